"""The operators for rounds of drafted trees and for windowed caches of callers' own models, as cases that can be timed and compared.

A case is one call on tensors that a program has in hand:

  window   attention of T new tokens over a paged cache, each seeing a window and a few first tokens (window_attn_static)
  tree     attention of a tree of drafted tokens over the paged cache they are part of (tree_attn_static)
  scores   log probabilities of given tokens, entropy and top alternatives, from logits (token_logprobs_static)
  walk     a tree of drafted tokens tested against the target's probabilities (verify_tree_static)
  keep     keys and values of the kept path moved together in the cache, all layers at once (keep_path_static)

Each has a plain form of elementary torch operations, which is what `run` computes unless `own` is set, and a definition in
64 bits.  Head sizes and counts are those of the workload configurations (16 heads of 64) and generic ones (grouped heads of
128), pages of 16 tokens as in the handles, or larger.
"""
import math

import torch

own = False
if own:
    import paper_2511_18191_amd as tsd  # noqa: F401

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # a decode step of one sequence behind a long history, all but the window and four first tokens dropped (latency)
        {"name": "window_one", "op": "window", "B": 1, "T": 1, "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "dtype": "bf16", "window": 1024, "sinks": 4,
         "least": 20000, "most": 20000},
        # one new token of a serving batch whose histories are shorter and longer than the window
        {"name": "window_batch", "op": "window", "B": 64, "T": 1, "Hq": 32, "Hkv": 8, "D": 128, "page": 16, "dtype": "bf16", "window": 4096, "sinks": 4,
         "least": 100, "most": 16384},
        # a chunk of two prompts behind what the cache holds of them
        {"name": "window_prompt", "op": "window", "B": 2, "T": 2048, "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "dtype": "bf16", "window": 1024, "sinks": 4,
         "least": 2048, "most": 8192},
        # a tree of 26 drafted tokens of one sequence (latency)
        {"name": "tree_one", "op": "tree", "B": 1, "T": 26, "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "dtype": "bf16", "window": 0, "sinks": 0,
         "least": 2000, "most": 2000, "ragged": False},
        # trees of all sizes of a small fp32 model with an odd head size, its layers windowed
        {"name": "tree_odd", "op": "tree", "B": 24, "T": 17, "Hq": 12, "Hkv": 4, "D": 80, "page": 16, "dtype": "fp32", "window": 500, "sinks": 3,
         "least": 1, "most": 1501, "ragged": True},
        # trees of 64 tokens of a serving batch, caches of all lengths
        {"name": "tree_batch", "op": "tree", "B": 16, "T": 64, "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "dtype": "bf16", "window": 0, "sinks": 0,
         "least": 500, "most": 16384, "ragged": False},
        # the score of one decoded token and five alternatives (latency)
        {"name": "scores_one", "op": "scores", "B": 1, "T": 1, "V": 32000, "dtype": "fp32", "top": 5, "temperature": 1.0, "ragged": False},
        # scores of sixteen tokens of every sequence, a large vocabulary, twenty alternatives
        {"name": "scores_batch", "op": "scores", "B": 64, "T": 16, "V": 131072, "dtype": "bf16", "top": 20, "temperature": 0.8, "ragged": False},
        # a tree of 26 tokens of one sequence
        {"name": "walk_one", "op": "walk", "B": 1, "N": 26, "V": 32000, "dtype": "fp32", "ragged": False},
        # trees of a serving batch, some of them smaller, an odd vocabulary
        {"name": "walk_batch", "op": "walk", "B": 64, "N": 32, "V": 50257, "dtype": "fp32", "ragged": True},
        # four kept tokens of one sequence in one layer's cache (latency)
        {"name": "keep_one", "op": "keep", "B": 1, "N": 26, "L": 1, "Hkv": 8, "D": 128, "page": 64, "dtype": "bf16", "kept": 4},
        # up to eight kept tokens of a serving batch, all layers of its cache
        {"name": "keep_batch", "op": "keep", "B": 64, "N": 64, "L": 24, "Hkv": 8, "D": 128, "page": 16, "dtype": "bf16", "kept": 8},
    ]


def _spread(rng, low, high):
    """A whole number between low and high, evenly over the logarithm."""
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    op = rng.choice(["window", "window", "tree", "tree", "scores", "scores", "walk", "keep"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    page = rng.choice([16, 32, 64])
    if op == "scores":
        B = _spread(rng, 1, 256)
        T = _spread(rng, 1, max(1, min(32, 1024 // B)))
        V = _spread(rng, 500, min(262144, (1024 * 131072) // (B * T) // (2 if dtype == "fp32" else 1)))
        return {"op": op, "B": B, "T": T, "V": V, "dtype": dtype, "top": rng.choice([0, 1, 5, 10, 20, 32]),
                "temperature": rng.choice([1.0, 1.0, 0.7, 1.3]), "ragged": rng.random() < 0.5}
    if op == "walk":
        B, N = _spread(rng, 1, 128), rng.randint(2, 64)
        V = _spread(rng, 500, min(131072, (64 * 32 * 50257) // (B * N)))
        return {"op": op, "B": B, "N": N, "V": V, "dtype": dtype, "ragged": rng.random() < 0.5}
    D = rng.choice([32, 64, 64, 80, 96, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8, 16])
    if op == "keep":
        B, N = _spread(rng, 1, 64), rng.randint(4, 64)
        return {"op": op, "B": B, "N": N, "L": _spread(rng, 1, 24), "Hkv": min(Hkv, 8), "D": D, "page": page, "dtype": dtype,
                "kept": rng.randint(1, min(8, N // 2))}
    Hq = Hkv * rng.choice([1, 2, 3, 4, 8] if Hkv <= 4 else [1, 2, 4])
    if op == "window":
        window, sinks = _spread(rng, 16, 4096), rng.choice([0, 1, 4, 4, 64])
        if rng.random() < 0.3:  # a chunk of prompts
            B, T = rng.randint(1, 2), _spread(rng, 18, 1024)
            most = _spread(rng, T, 8192)
            window = min(window, 1024)
        else:
            B, T = _spread(rng, 1, 256), rng.randint(1, 9)
            window = min(window, (64 * 4096) // B)
            most = _spread(rng, 8, 16384)
        return {"op": op, "B": B, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "dtype": dtype, "window": window, "sinks": sinks,
                "least": rng.randint(1, most), "most": most}
    B, T = _spread(rng, 1, 64), rng.randint(2, 64)
    most = _spread(rng, 8, max(8, min(16384, (16 * 16384) // B)))
    windowed = rng.random() < 0.3
    return {"op": op, "B": B, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "dtype": dtype, "window": _spread(rng, 16, 4096) if windowed else 0,
            "sinks": rng.choice([0, 4]) if windowed else 0, "least": rng.randint(1, most), "most": most, "ragged": rng.random() < 0.5}


# ---- inputs ---------------------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & 0x7FFFFFFF)
    return g


def _counts(case, most, g):
    """How many new tokens of a sequence are there (int32 [B])."""
    if not case["ragged"]:
        return torch.full((case["B"],), most, device=DEV, dtype=torch.int32)
    return torch.randint(0, most + 1, (case["B"],), device=DEV, generator=g).to(torch.int32)


DEEP = 8  # levels of a tree below its root


def _trees(B, N, g):
    """Parents of N nodes in topological order, int32 [B, N]: node 0 is the root, another hangs on one of the eight before it, or on
    the root where that lies DEEP levels down."""
    n = torch.arange(N, device=DEV)
    up = n - 1 - (torch.rand(B, N, device=DEV, generator=g) * n.clamp(max=8)).long()
    depth = torch.zeros(B, N, dtype=torch.long, device=DEV)
    for i in range(1, N):
        above = depth.gather(1, up[:, i:i + 1])[:, 0]
        up[:, i] = torch.where(above < DEEP, up[:, i], 0)
        depth[:, i] = torch.where(above < DEEP, above + 1, 1)
    return up.to(torch.int32)


def prepare(case, seed):
    g = _generator(seed)
    dt = TYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "scores":
        B, T, V = case["B"], case["T"], case["V"]
        s["logits"] = torch.randn(B, T, V, device=DEV, generator=g, dtype=dt if B * T * V > 1 << 24 else torch.float32).mul_(3.0).to(dt)
        s["tokens"] = torch.randint(0, V, (B, T), device=DEV, generator=g)
        s["n_new"] = _counts(case, T, g) if case["ragged"] else None
        return s
    if case["op"] == "walk":
        B, N, V = case["B"], case["N"], case["V"]
        p = torch.softmax(5.0 * torch.randn(B, N, V, device=DEV, generator=g), -1)
        parents = _trees(B, N, g)
        # a node's children are the likeliest tokens behind it, as a good draft finds them: half of the steps find theirs
        up = parents.long().clamp(min=0)
        likely = p.topk(8, -1).indices
        born = torch.zeros(B, N, dtype=torch.long, device=DEV)
        for n in range(1, N):
            born[:, n] = (parents[:, 1:n] == parents[:, n:n + 1]).sum(1)
        each = torch.arange(B, device=DEV)[:, None]
        s["tokens"] = likely[each, up, born.clamp(max=7)].to(torch.int32)
        s["p"], s["parents"] = p.to(dt), parents
        s["uniforms"] = torch.rand(B, N, device=DEV, generator=g)
        s["n_new"] = _counts(case, N - 1, g) + 1 if case["ragged"] else None
        return s
    page, Hkv, D, B = case["page"], case["Hkv"], case["D"], case["B"]
    if case["op"] == "keep":
        N, L, m = case["N"], case["L"], case["kept"]
        cols = -(-(200 + N) // page)
        shape = (L, B * cols, page, Hkv, D)
        s["k_pool"], s["v_pool"] = (torch.randn(shape, device=DEV, generator=g, dtype=dt) for _ in range(2))
        s["table"] = torch.randperm(B * cols, device=DEV, generator=g).to(torch.int32).view(B, cols)
        s["held"] = torch.randint(0, 201, (B,), device=DEV, generator=g).to(torch.int32)
        # the root, then nodes behind those that the path moves to
        order = torch.argsort(torch.rand(B, N - m, device=DEV, generator=g), 1)[:, :m - 1].sort(1).values + m
        kept = torch.randint(1, m + 1, (B, 1), device=DEV, generator=g) if B > 1 else torch.full((B, 1), m, device=DEV)
        path = torch.full((B, N), -1, device=DEV, dtype=torch.int32)
        path[:, 0] = 0
        path[:, 1:m] = torch.where(torch.arange(1, m, device=DEV)[None] < kept, order, -1).to(torch.int32)
        s["path"] = path
        return s
    T, most, window, sinks = case["T"], case["most"], case["window"], case["sinks"]
    lens = torch.randint(case["least"], most + 1, (B,), device=DEV, generator=g)
    n_new = torch.minimum(lens, torch.full_like(lens, T))  # a cache shorter than T holds fewer new tokens
    if case["op"] == "tree":
        n_new = torch.minimum(lens, _counts(case, T, g).long())
        s["parents"] = _trees(B, T, g)
    # the cache keeps the pages of the first tokens and of the window, dealt out in no order; the others were dropped
    cols = -(-most // page)
    col = torch.arange(cols, device=DEV)[None]
    first = ((lens - n_new - window + 1).clamp(min=0) if window else torch.zeros_like(lens))[:, None]
    kept = ((col + 1) * page > first) | (col * page < sinks)
    kept &= col * page < lens[:, None]
    pages = B * min(cols, -(-(window + T) // page) + 1 + -(-sinks // page)) if window else B * cols
    order = torch.randperm(pages, device=DEV, generator=g)
    s["table"] = torch.where(kept, order[(kept.flatten().cumsum(0) - 1).clamp(min=0)].view(B, cols), -1).to(torch.int32)
    s["k_pool"], s["v_pool"] = (torch.randn(pages, page, Hkv, D, device=DEV, generator=g).to(dt) for _ in range(2))
    s["q"] = (1.5 * torch.randn(B, T, case["Hq"], D, device=DEV, generator=g)).to(dt)
    s["lens"], s["n_new"] = lens.to(torch.int32), n_new.to(torch.int32)
    s["out"] = torch.zeros(B, T, case["Hq"], D, device=DEV, dtype=dt)
    return s


# ---- the operators --------------------------------------------------------------------------------------------------------------

def run(s):
    case, op = s["case"], s["case"]["op"]
    if own:
        import paper_2511_18191_amd as tsd
        if op == "window":
            return tsd.window_attn_static(s["q"], s["k_pool"], s["v_pool"], s["table"], s["lens"], case["window"], sinks=case["sinks"],
                                          max_len=case["most"], n_new=s["n_new"], out=s["out"])
        if op == "tree":
            return tsd.tree_attn_static(s["q"], s["k_pool"], s["v_pool"], s["table"], s["lens"], s["parents"], window=case["window"] or None,
                                        sinks=case["sinks"], max_len=case["most"], n_new=s["n_new"], out=s["out"])
        if op == "scores":
            got = tsd.token_logprobs_static(s["logits"], s["tokens"], top=case["top"], temperature=case["temperature"], n_new=s["n_new"])
            return [got["logprobs"], got["entropy"]] + ([got["top_ids"], got["top_logprobs"]] if case["top"] else [])
        if op == "walk":
            got = tsd.verify_tree_static(s["tokens"], s["parents"], p=s["p"], uniforms=s["uniforms"], n_new=s["n_new"])
            return [got["n_acc"], got["tokens"], got["path"]]
        tsd.keep_path_static(s["k_pool"], s["v_pool"], s["table"], s["held"], s["path"])
        return [s["k_pool"], s["v_pool"]]
    return {"window": _attn, "tree": _attn, "scores": _scores, "walk": _walk, "keep": _keep}[op](s)


def _depths(parents):
    """Depth of every node, [B, N], and whether node j is node i or among its ancestors, [B, N, N]."""
    B, N = parents.shape
    line = torch.eye(N, device=parents.device, dtype=torch.bool).expand(B, N, N).clone()
    for n in range(1, N):
        up = parents[:, n].long()
        above = line.gather(1, up.clamp(min=0)[:, None, None].expand(B, 1, N))[:, 0]
        line[:, n] |= above & (up >= 0)[:, None]
    return line.sum(-1) - 1, line


def _attn(s):
    case, q, lens, n_new = s["case"], s["q"], s["lens"].long(), s["n_new"].long()
    B, T, Hq, D = q.shape
    Hkv, page, window, sinks = case["Hkv"], case["page"], case["window"] or 1 << 30, case["sinks"]
    held, step = lens - n_new, torch.arange(T, device=q.device)
    # the slots that some token sees: the first ones, and those from the first token's window on
    wide = min(case["most"], window + T)
    first = torch.maximum((held - window + 1).clamp(min=0), (lens - wide).clamp(min=0))
    slots = torch.cat([torch.arange(sinks, device=q.device).expand(B, sinks), first[:, None] + torch.arange(wide, device=q.device)], 1)
    there = slots < lens[:, None]
    there[:, :sinks] &= slots[:, :sinks] < first[:, None]
    at = s["table"].long().gather(1, (slots // page).clamp(max=s["table"].shape[1] - 1))
    there &= at >= 0
    at, row = at.clamp(min=0), slots % page
    k = s["k_pool"][at, row].float().transpose(1, 2)  # [B, Hkv, slots, D]
    v = s["v_pool"][at, row].float().transpose(1, 2)
    rows = q.float().view(B, T, Hkv, Hq // Hkv, D).transpose(1, 2).reshape(B, Hkv, T * (Hq // Hkv), D)
    scores = torch.matmul(rows, k.transpose(2, 3).contiguous()) / math.sqrt(D)
    j = slots[:, None]  # [B, 1, slots]
    if case["op"] == "tree":
        depth, line = _depths(s["parents"])
        node = (j - held[:, None, None]).clamp(0, T - 1)  # of the keys that are nodes
        is_node = j >= held[:, None, None]
        place = held[:, None, None] + depth[:, :, None]
        of_key = torch.where(is_node, held[:, None, None] + depth[:, None].gather(2, node), j)
        sees = torch.where(is_node, line.gather(2, node.expand(B, T, -1)), torch.ones_like(is_node))
    else:
        place, of_key = (held[:, None] + step)[:, :, None], j
        sees = j <= place
    sees = sees & ((of_key > place - window) | (of_key < sinks)) & there[:, None]
    scores = torch.where(sees.repeat_interleave(Hq // Hkv, 1)[:, None], scores, -math.inf)
    weights = torch.exp(scores - scores.amax(-1, keepdim=True).clamp(min=-3e38))
    total = weights.sum(-1, keepdim=True)
    out = torch.matmul(weights, v) / torch.where(total > 0, total, 1.0)
    out = out.view(B, Hkv, T, Hq // Hkv, D).transpose(1, 2).reshape(B, T, Hq, D).to(q.dtype)
    s["out"].copy_(torch.where((step < n_new[:, None])[..., None, None], out, s["out"]))
    return s["out"]


def _scores(s):
    case, logits, tokens = s["case"], s["logits"], s["tokens"]
    B, T, V = logits.shape
    x = logits.float() / case["temperature"]
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    lse = top + total.log()
    there = torch.arange(T, device=x.device)[None] < (s["n_new"][:, None] if s["n_new"] is not None else T)
    entropy = total.log()[..., 0] - (e * (x - top)).sum(-1) / total[..., 0]
    outs = [torch.where(there, (x.gather(2, tokens[..., None]) - lse)[..., 0], 0.0), torch.where(there, entropy, 0.0)]
    if case["top"]:
        # by value, the lowest index first: whole numbers in the values' order, the index behind them
        bits = logits.float().view(torch.int32).long()
        key = torch.where(bits >= 0, bits, bits ^ 0x7FFFFFFF) * (1 << 20) + (V - 1 - torch.arange(V, device=x.device))
        best = key.topk(case["top"], -1).indices
        outs += [torch.where(there[..., None], best, -1).to(torch.int32), torch.where(there[..., None], x.gather(2, best) - lse, 0.0)]
    return outs


def _walk(s):
    tokens, parents, p, u = s["tokens"].long(), s["parents"].long(), s["p"], s["uniforms"].double()
    B, N = tokens.shape
    nodes = s["n_new"].long() if s["n_new"] is not None else torch.full((B,), N, device=p.device)
    series, node = torch.arange(B, device=p.device), torch.arange(N, device=p.device)[None]
    at, going = torch.zeros_like(nodes), torch.ones_like(nodes, dtype=torch.bool)
    n_acc = torch.zeros_like(nodes)
    out, path = torch.full((B, N), -1, device=p.device, dtype=torch.long), torch.full((B, N), -1, device=p.device, dtype=torch.long)
    path[:, 0] = 0
    for i in range(min(N, DEEP + 1)):
        # (64 bits: a draw next to a border between two tokens goes by the last bits of the sums)
        sums = p[series, at].double().cumsum(1)
        token = (sums <= u[:, i:i + 1] * sums[:, -1:]).sum(1)
        out[:, i] = torch.where(going, token, out[:, i])
        fits = (parents == at[:, None]) & (tokens == token[:, None]) & (node > at[:, None]) & (node < nodes[:, None])
        going = going & fits.any(1)
        at = torch.where(going, torch.where(fits, node, N).amin(1), at)
        n_acc += going
        if i + 1 < N:
            path[:, i + 1] = torch.where(going, at, -1)
    return [n_acc.to(torch.int32), out.to(torch.int32), path.to(torch.int32)]


def _keep(s):
    case, path, held, page = s["case"], s["path"].long(), s["held"].long(), s["case"]["page"]
    m = case["kept"]
    kept = path[:, :m] >= 0
    to = held[:, None] + torch.arange(m, device=path.device)
    source = torch.where(kept, held[:, None] + path[:, :m], to)  # (what is not kept stays)
    at = [(s["table"].long().gather(1, x // page), x % page) for x in (source, to)]
    for pool in (s["k_pool"], s["v_pool"]):
        pool[:, at[1][0], at[1][1]] = pool[:, at[0][0], at[0][1]]
    return [s["k_pool"], s["v_pool"]]


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"window": _exact_attn, "tree": _exact_attn, "scores": _exact_scores, "walk": _exact_walk, "keep": _exact_keep}[case["op"]](s)


def _exact_attn(s):
    case, out = s["case"], s["out"].double()
    D, group, page = case["D"], case["Hq"] // case["Hkv"], case["page"]
    window, sinks = case["window"] or 1 << 30, case["sinks"]
    parents = s["parents"].tolist() if case["op"] == "tree" else None
    for b, (length, n) in enumerate(zip(s["lens"].tolist(), s["n_new"].tolist())):
        held = length - n
        place = [*range(held), *[held + t for t in range(n)]]  # of every slot
        sees = torch.ones(n, length, dtype=torch.bool)
        if parents:
            depth = []
            sees[:, held:] = False
            for t in range(n):
                a = parents[b][t]
                depth.append(depth[a] + 1 if a >= 0 else 0)
                place[held + t] = held + depth[t]
                if a >= 0:
                    sees[t] |= sees[a]
                sees[t, held + t] = True
        else:
            sees = torch.tril(sees, held)
        place = torch.tensor(place)
        sees &= (place[None] > place[held:, None] - window) | (place[None] < sinks)
        sees &= (s["table"][b].cpu() >= 0).repeat_interleave(page)[:length]
        used = sees.any(0).nonzero()[:, 0].to(DEV)
        if not n or not len(used):
            continue
        mask = sees.to(DEV)[:, used].repeat_interleave(group, 0)
        rows = s["table"][b].long()[used // page] * page + used % page
        for h in range(case["Hkv"]):
            k, v = (x.view(-1, *x.shape[2:])[rows, h].double() for x in (s["k_pool"], s["v_pool"]))
            scores = s["q"][b, :n, h * group:(h + 1) * group].double().reshape(-1, D) @ k.T.contiguous() / D ** 0.5
            out[b, :n, h * group:(h + 1) * group] = (torch.softmax(scores.masked_fill_(~mask, -math.inf), -1) @ v).view(n, group, D)
    return out


def _exact_scores(s):
    case, n_new = s["case"], s["n_new"].tolist() if s["n_new"] is not None else [s["case"]["T"]] * s["case"]["B"]
    B, T, k = case["B"], case["T"], case["top"]
    outs = [torch.zeros(B, T, dtype=torch.float64), torch.zeros(B, T, dtype=torch.float64)]
    if k:
        outs += [torch.full((B, T, k), -1, dtype=torch.int32), torch.zeros(B, T, k, dtype=torch.float64)]
    for b in range(B):
        for t in range(n_new[b]):
            row = s["logits"][b, t].double()
            lp = torch.log_softmax(row / case["temperature"], 0)
            outs[0][b, t] = lp[s["tokens"][b, t]]
            outs[1][b, t] = -(lp.exp() * lp).sum()
            if k:
                best = torch.sort(row, descending=True, stable=True).indices[:k]
                outs[2][b, t], outs[3][b, t] = best, lp[best]
    return outs


def _exact_walk(s):
    B, N = s["tokens"].shape
    tokens, parents, u = s["tokens"].tolist(), s["parents"].tolist(), s["uniforms"].double().tolist()
    nodes = s["n_new"].tolist() if s["n_new"] is not None else [N] * B
    n_acc, out, path = [], [], []
    for b in range(B):
        at, drawn, way = 0, [], [0]
        while True:
            sums = torch.cumsum(s["p"][b, at].double().cpu(), 0)
            drawn.append(int(torch.searchsorted(sums, u[b][len(drawn)] * float(sums[-1]), right=True)))
            at = next((c for c in range(at + 1, nodes[b]) if parents[b][c] == at and tokens[b][c] == drawn[-1]), -1)
            if at < 0:
                break
            way.append(at)
        n_acc.append(len(way) - 1)
        out.append(drawn + [-1] * (N - len(drawn)))
        path.append(way + [-1] * (N - len(way)))
    return [torch.tensor(x, dtype=torch.int32) for x in (n_acc, out, path)]


def _exact_keep(s):
    page, outs = s["case"]["page"], []
    for pool in (s["k_pool"], s["v_pool"]):
        old, new = pool, pool.double()
        for b, (held, path) in enumerate(zip(s["held"].tolist(), s["path"].tolist())):
            for i, n in enumerate(path):
                if n >= 0:
                    x, y = held + n, held + i
                    new[:, s["table"][b, y // page].long(), y % page] = old[:, s["table"][b, x // page].long(), x % page].double()
        outs.append(new)
    return outs


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    B = case["B"]
    if case["op"] == "scores":
        rows = B * case["T"] / (2 if case["ragged"] else 1)
        return {"bytes": rows * (case["V"] * size + 16 + 8 * case["top"]), "flops": 6 * rows * case["V"]}
    if case["op"] == "walk":
        steps = 2  # (rows of probabilities on the way: half of the steps find a child)
        return {"bytes": B * (steps * case["V"] * size + 20 * case["N"]), "flops": 2 * B * steps * case["V"]}
    row = case["Hkv"] * case["D"] * size
    if case["op"] == "keep":
        moved = B * (case["kept"] - 1) / (2 if B > 1 else 1)
        return {"bytes": moved * case["L"] * row * 4, "flops": 0}
    T, Hq, window, sinks = case["T"], case["Hq"], case["window"] or 1 << 30, case["sinks"]
    keys = pairs = news = 0.0
    for i in range(32):  # the lengths evenly between the least and the most
        length = case["least"] + (case["most"] - case["least"]) * (i + 0.5) / 32
        n = min(length, T / 2 if case.get("ragged") else T)
        seen = min(length, window + sinks)
        keys += min(length, seen + n - 1) / 32
        news += n / 32
        pairs += n * (min(seen, length - (n - 1) / 2) if case["op"] == "window" else min(seen, length - n + min(n, 6))) / 32
    return {"bytes": B * (2 * keys * row + 2 * news * Hq * case["D"] * size), "flops": 4 * B * pairs * Hq * case["D"]}
