"""The operators for callers' own models, as cases that can be timed and compared.

A case is one call on tensors that a program has in hand:

  append   rotary positions on queries and keys, keys and values written into a paged cache (rope_append_static)
  attn     attention of T new tokens over the paged cache they are part of (paged_attn_static)
  verify   drafted tokens tested against the target's probabilities, the residual draw (verify_tokens_static)

Each has a plain form of elementary torch operations, which is what `run` computes unless `own` is set, and a definition in
64 bits.  Head sizes and counts are those of the workload configurations (8 to 16 heads of 64) and generic ones (grouped
heads of 128), pages of 16 tokens as in the handles, or larger.
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
        # a decode step of one series: 16 heads of 64, whole head rotated in halves (latency)
        {"name": "append_one", "op": "append", "B": 1, "T": 1, "Hq": 16, "Hkv": 16, "D": 64, "R": 64, "page": 16, "dtype": "bf16",
         "pairs": "half", "scaling": "none", "start": 60, "ragged": False},
        # the pending token and four proposals of a ragged batch, neighbouring dims paired, part of an odd-sized head, far positions
        {"name": "append_odd", "op": "append", "B": 93, "T": 5, "Hq": 12, "Hkv": 4, "D": 80, "R": 32, "page": 16, "dtype": "fp32",
         "pairs": "interleaved", "scaling": "linear", "start": 100000, "ragged": True},
        # the prompts of four sequences at once, frequencies blended for long contexts
        {"name": "append_prompts", "op": "append", "B": 4, "T": 4096, "Hq": 32, "Hkv": 8, "D": 128, "R": 128, "page": 64, "dtype": "bf16",
         "pairs": "half", "scaling": "blend", "start": 0, "ragged": False},
        # a decode step of one series over a history of 60 patches (latency)
        {"name": "attn_one", "op": "attn", "B": 1, "T": 1, "Hq": 16, "Hkv": 16, "D": 64, "page": 16, "dtype": "bf16", "least": 61, "most": 61},
        # verification of four proposals of one sequence over a long cache: few rows, split over the length
        {"name": "attn_long", "op": "attn", "B": 1, "T": 5, "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "dtype": "bf16", "least": 32768, "most": 32768},
        # one new token of a serving batch whose caches are of all lengths
        {"name": "attn_batch", "op": "attn", "B": 64, "T": 1, "Hq": 32, "Hkv": 8, "D": 128, "page": 16, "dtype": "bf16", "least": 100, "most": 8192},
        # verification of six proposals of a large batch, short histories, a key head per query head
        {"name": "attn_many", "op": "attn", "B": 512, "T": 7, "Hq": 16, "Hkv": 16, "D": 64, "page": 16, "dtype": "bf16", "least": 70, "most": 90},
        # an fp32 model with an odd head size and a ragged number of proposals
        {"name": "attn_odd", "op": "attn", "B": 6, "T": 3, "Hq": 12, "Hkv": 4, "D": 80, "page": 16, "dtype": "fp32", "least": 1, "most": 1501},
        # a chunk of two prompts behind what the cache holds of them
        {"name": "attn_prompt", "op": "attn", "B": 2, "T": 1024, "Hq": 32, "Hkv": 8, "D": 128, "page": 64, "dtype": "bf16", "least": 2048, "most": 4096},
        # four drafts of one sequence
        {"name": "verify_one", "op": "verify", "B": 1, "K": 4, "V": 32000, "dtype": "fp32", "ragged": False},
        # six drafts of a serving batch over a large vocabulary
        {"name": "verify_batch", "op": "verify", "B": 64, "K": 6, "V": 131072, "dtype": "fp32", "ragged": False},
        # ragged drafts of many sequences, an odd vocabulary, probabilities in 16 bits
        {"name": "verify_many", "op": "verify", "B": 256, "K": 8, "V": 50257, "dtype": "bf16", "ragged": True},
    ]


def _spread(rng, low, high):
    """A whole number between low and high, evenly over the logarithm."""
    return min(high, max(low, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    op = rng.choice(["append", "attn", "attn", "verify"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    page = rng.choice([16, 32, 64])
    if op == "verify":
        B, K = _spread(rng, 1, 256), rng.randint(1, 12)
        V = _spread(rng, 500, min(131072, (64 * 6 * 131072) // (B * K)))
        return {"op": op, "B": B, "K": K, "V": V, "dtype": dtype, "ragged": rng.random() < 0.5}
    D = rng.choice([32, 64, 64, 80, 96, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8, 16])
    Hq = Hkv * rng.choice([1, 2, 3, 4, 8] if Hkv <= 4 else [1, 2, 4])
    if op == "append":
        B = _spread(rng, 1, 512)
        T = _spread(rng, 1, max(1, min(4096, 16384 // B)))
        return {"op": op, "B": B, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "R": rng.choice([D, D, D // 2]), "page": page, "dtype": dtype,
                "pairs": rng.choice(["half", "interleaved"]), "scaling": rng.choice(["none", "linear", "base", "blend"]),
                "start": _spread(rng, 1, 100000), "ragged": rng.random() < 0.5}
    if rng.random() < 0.2:  # a chunk of prompts
        B, T = rng.randint(1, 2), _spread(rng, 18, 1024)
        most = _spread(rng, T, 4096)
        return {"op": op, "B": B, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "dtype": dtype, "least": rng.randint(1, most), "most": most}
    B, T = _spread(rng, 1, 512), rng.randint(1, 9)
    most = _spread(rng, 8, max(8, min(32768, (64 * 8192) // B)))
    return {"op": op, "B": B, "T": T, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "dtype": dtype, "least": rng.randint(1, most), "most": most}


# ---- inputs ---------------------------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & 0x7FFFFFFF)
    return g


def _paged(case, cols, g, zero):
    """Pools and a page table that deals their pages out in no order."""
    n = case["B"] * cols
    shape = (n, case["page"], case["Hkv"], case["D"])
    make = (lambda: torch.zeros(shape, device=DEV, dtype=TYPES[case["dtype"]])) if zero else (
        lambda: torch.randn(shape, device=DEV, generator=g).to(TYPES[case["dtype"]]))
    table = torch.randperm(n, device=DEV, generator=g).to(torch.int32).view(case["B"], cols)
    return make(), make(), table


def _frequencies(case):
    """The rotary frequencies (radians per position) and the amplitude: what the framework's rope_frequencies gives, by hand."""
    R, base, factor = case["R"], 10000.0, 8.0
    i = torch.arange(0, R, 2, dtype=torch.float64)
    if case["scaling"] == "base":
        base = base * factor ** (R / (R - 2))
    f = base ** (-i / R)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] != "blend":
        return f.to(DEV), 1.0
    keep = ((4096 * f / (2 * math.pi) - 1.0) / (32.0 - 1.0)).clamp(0, 1)
    return (f * (keep + (1 - keep) / factor)).to(DEV), 0.1 * math.log(factor) + 1.0


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] == "verify":
        B, K, V, dt = case["B"], case["K"], case["V"], TYPES[case["dtype"]]
        # the draft's logits are the target's with noise: some 0.8 of the drafts pass
        logits = 2.5 * torch.randn(B, K + 1, V, device=DEV, generator=g)
        p = torch.softmax(logits, -1).to(dt)
        noisy = logits[:, :K] + 0.5 * torch.randn(B, K, V, device=DEV, generator=g)
        del logits
        q = torch.softmax(noisy, -1).to(dt)
        noisy -= torch.log(-torch.log(torch.rand(B, K, V, device=DEV, generator=g).clamp(1e-12, 1 - 1e-7)))
        draft = noisy.argmax(-1).to(torch.int32)
        del noisy
        uniforms = torch.rand(B, K + 1, device=DEV, generator=g)
        n_draft = torch.randint(0, K + 1, (B,), device=DEV, generator=g).to(torch.int32) if case["ragged"] else None
        return {"case": case, "draft": draft, "q": q, "p": p, "uniforms": uniforms, "n_draft": n_draft}
    B, T, Hq, Hkv, D, page = (case[k] for k in ("B", "T", "Hq", "Hkv", "D", "page"))
    dt = TYPES[case["dtype"]]
    new = lambda h: torch.randn(B, T, h, D, device=DEV, generator=g).to(dt)
    if case["op"] == "append":
        # sequences whose positions go on from `start` and less; their caches hold the last up to 200 tokens before the new ones
        held = torch.randint(0, min(200, case["start"]) + 1, (B,), device=DEV, generator=g).to(torch.int32)
        first = torch.randint(case["start"] // 2, case["start"] + 1, (B,), device=DEV, generator=g)
        positions = (first[:, None] + torch.arange(T, device=DEV)[None]).to(torch.int32)
        k_pool, v_pool, table = _paged(case, -(-(200 + T) // page), g, True)
        n_new = torch.randint(0, T + 1, (B,), device=DEV, generator=g).to(torch.int32) if case["ragged"] else None
        freq, amplitude = _frequencies(case)
        return {"case": case, "q": new(Hq), "k": new(Hkv), "v": new(Hkv), "k_pool": k_pool, "v_pool": v_pool, "table": table, "held": held,
                "positions": positions, "n_new": n_new, "freq": freq, "amplitude": amplitude, "out": torch.zeros(B, T, Hq, D, device=DEV, dtype=dt)}
    lens = torch.randint(case["least"], case["most"] + 1, (B,), device=DEV, generator=g).to(torch.int32)
    k_pool, v_pool, table = _paged(case, -(-case["most"] // page), g, False)
    n_new = torch.minimum(lens, torch.full_like(lens, T))  # a cache shorter than T holds fewer new tokens
    return {"case": case, "q": 1.5 * new(Hq), "k_pool": k_pool, "v_pool": v_pool, "table": table, "lens": lens, "n_new": n_new,
            "out": torch.zeros(B, T, Hq, D, device=DEV, dtype=dt)}


# ---- the operators --------------------------------------------------------------------------------------------------------------

def run(s):
    op = s["case"]["op"]
    if own:
        import paper_2511_18191_amd as tsd
        if op == "append":
            tsd.rope_append_static(s["q"], s["k"], s["v"], s["k_pool"], s["v_pool"], s["table"], s["held"], s["freq"], positions=s["positions"],
                                   n_new=s["n_new"], interleaved=s["case"]["pairs"] == "interleaved", amplitude=s["amplitude"], out=s["out"])
            return [s["out"], s["k_pool"], s["v_pool"]]
        if op == "attn":
            return tsd.paged_attn_static(s["q"], s["k_pool"], s["v_pool"], s["table"], s["lens"], max_len=s["case"]["most"], n_new=s["n_new"],
                                         out=s["out"])
        got = tsd.verify_tokens_static(s["draft"], s["q"], s["p"], s["uniforms"], n_draft=s["n_draft"])
        return [got["n_acc"], got["tokens"]]
    return {"append": _append, "attn": _attn, "verify": _verify}[op](s)


def _rotated(x, cos, sin, interleaved):
    R = 2 * cos.shape[-1]
    y = x[..., :R].float()
    a, b = (y[..., 0::2], y[..., 1::2]) if interleaved else (y[..., :R // 2], y[..., R // 2:])
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned.to(x.dtype), x[..., R:]], -1)


def _append(s):
    q, table, held, page = s["q"], s["table"], s["held"], s["case"]["page"]
    B, T = q.shape[:2]
    angle = s["positions"].double()[:, :, None, None] * s["freq"]  # (64 bits: far positions lose their fraction of a turn in 32)
    cos, sin = (s["amplitude"] * angle.cos()).float(), (s["amplitude"] * angle.sin()).float()
    interleaved = s["case"]["pairs"] == "interleaved"
    step = torch.arange(T, device=q.device)[None]
    there = (step < (s["n_new"][:, None] if s["n_new"] is not None else T)).expand(B, T)[:, :, None, None]
    slot = held.long()[:, None] + step
    at, row = table.gather(1, slot // page).long(), slot % page
    s["k_pool"][at, row] = torch.where(there, _rotated(s["k"], cos, sin, interleaved), s["k_pool"][at, row])
    s["v_pool"][at, row] = torch.where(there, s["v"], s["v_pool"][at, row])
    s["out"].copy_(torch.where(there, _rotated(q, cos, sin, interleaved), s["out"]))
    return [s["out"], s["k_pool"], s["v_pool"]]


def _attn(s):
    q, lens, n_new, most = s["q"], s["lens"], s["n_new"], s["case"]["most"]
    B, T, Hq, D = q.shape
    Hkv = s["k_pool"].shape[2]
    pages = s["table"].long()
    k = s["k_pool"][pages].flatten(1, 2)[:, :most].float().transpose(1, 2)  # [B, Hkv, most, D]
    v = s["v_pool"][pages].flatten(1, 2)[:, :most].float().transpose(1, 2)
    rows = q.float().view(B, T, Hkv, Hq // Hkv, D).transpose(1, 2).reshape(B, Hkv, T * (Hq // Hkv), D)
    scores = torch.matmul(rows, k.transpose(2, 3).contiguous()) / math.sqrt(D)
    step = torch.arange(T, device=q.device)[None, :, None]
    sees = torch.arange(most, device=q.device)[None, None] < (lens - n_new)[:, None, None] + step + 1  # [B, T, most]
    sees &= torch.arange(most, device=q.device)[None, None] < lens[:, None, None]
    sees = sees.repeat_interleave(Hq // Hkv, 1)[:, None]
    scores = torch.where(sees, scores, -math.inf)
    weights = torch.exp(scores - scores.amax(-1, keepdim=True).clamp(min=-3e38))
    out = torch.matmul(weights, v) / weights.sum(-1, keepdim=True)
    out = out.view(B, Hkv, T, Hq // Hkv, D).transpose(1, 2).reshape(B, T, Hq, D).to(q.dtype)
    there = (step < n_new[:, None, None])[..., None]
    s["out"].copy_(torch.where(there, out, s["out"]))
    return s["out"]


def _verify(s):
    draft, q, p, u = s["draft"], s["q"], s["p"], s["uniforms"].double()
    B, K = draft.shape
    at = draft.long()[..., None]
    of_p, of_q = p[:, :K].gather(2, at)[..., 0].double(), q.gather(2, at)[..., 0].double()
    drafted = s["n_draft"].long() if s["n_draft"] is not None else torch.full((B,), K, device=draft.device)
    step = torch.arange(K + 1, device=draft.device)[None]
    passed = (u[:, :K] * of_q < of_p) & (step[:, :K] < drafted[:, None])
    n = passed.long().cumprod(1).sum(1)
    series = torch.arange(B, device=draft.device)
    row_p, row_q = p[series, n].double(), q[series, n.clamp(max=K - 1)].double()
    # (64 bits: a draw next to a border between two tokens goes by the last bits of the sums)
    rest = torch.where((n < drafted)[:, None], (row_p - row_q).clamp(min=0), row_p)
    rest = torch.where(rest.sum(1, keepdim=True) > 0, rest, row_p)
    sums = rest.cumsum(1)
    token = (sums <= u[:, K:] * sums[:, -1:]).sum(1)
    tokens = torch.where(step < n[:, None], torch.cat([draft.long(), draft[:, :1].long()], 1), torch.where(step == n[:, None], token[:, None], -1))
    return [n.to(torch.int32), tokens.to(torch.int32)]


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attn": _exact_attn, "verify": _exact_verify}[case["op"]](s)


def _exact_append(s):
    case, page = s["case"], s["case"]["page"]
    B, T, R = case["B"], case["T"], case["R"]
    turn = torch.polar(torch.full((), s["amplitude"], dtype=torch.float64, device=DEV), s["positions"].double()[..., None] * s["freq"])

    def turned(x):
        y = x.double().clone()
        if case["pairs"] == "interleaved":
            z = torch.view_as_complex(y[..., :R].reshape(*y.shape[:-1], R // 2, 2).contiguous())
            y[..., :R] = torch.view_as_real(z * turn[:, :, None]).flatten(-2)
        else:
            z = torch.complex(y[..., :R // 2], y[..., R // 2:R]) * turn[:, :, None]
            y[..., :R // 2], y[..., R // 2:R] = z.real, z.imag
        return y

    out, k_pool, v_pool = s["out"].double(), s["k_pool"].double(), s["v_pool"].double()
    q, k = turned(s["q"]), turned(s["k"])
    table, held = s["table"].cpu(), s["held"].tolist()
    counts = s["n_new"].tolist() if s["n_new"] is not None else [T] * B
    for b in range(B):
        n = counts[b]
        out[b, :n] = q[b, :n]
        slots = torch.arange(held[b], held[b] + n)
        at = (table[b, slots // page].long() * page + slots % page).to(DEV)
        k_pool.view(-1, *k.shape[2:])[at] = k[b, :n]
        v_pool.view(-1, *k.shape[2:])[at] = s["v"][b, :n].double()
    return [out, k_pool, v_pool]


def _exact_attn(s):
    out, group = s["out"].double(), s["case"]["Hq"] // s["case"]["Hkv"]
    D, T = s["case"]["D"], s["case"]["T"]
    for b, (length, n) in enumerate(zip(s["lens"].tolist(), s["n_new"].tolist())):
        pages = s["table"][b].long()
        k, v = (x[pages].reshape(-1, *x.shape[2:])[:length].double() for x in (s["k_pool"], s["v_pool"]))
        for h in range(s["case"]["Hkv"]):
            q = s["q"][b, :n, h * group:(h + 1) * group].double()  # [n, group, D]
            scores = q.reshape(-1, D) @ k[:, h].T.contiguous() / D ** 0.5
            last = length - n + torch.arange(n, device=DEV).repeat_interleave(group)
            scores.masked_fill_(torch.arange(length, device=DEV)[None] > last[:, None], -math.inf)
            out[b, :n, h * group:(h + 1) * group] = (torch.softmax(scores, -1) @ v[:, h].contiguous()).view(n, group, D)
    return out


def _exact_verify(s):
    B, K = s["draft"].shape
    p, q, u, draft = s["p"], s["q"], s["uniforms"].double().tolist(), s["draft"].tolist()
    drafted = s["n_draft"].tolist() if s["n_draft"] is not None else [K] * B
    near = s["draft"].long()[..., None]
    of_p, of_q = p[:, :K].gather(2, near)[..., 0].double().tolist(), q.gather(2, near)[..., 0].double().tolist()
    n_acc, tokens = [], []
    for b in range(B):
        n = 0
        while n < drafted[b] and u[b][n] * of_q[b][n] < of_p[b][n]:
            n += 1
        weights = p[b, n].double().cpu()
        if n < drafted[b]:
            rest = torch.relu(weights - q[b, n].double().cpu())
            weights = rest if float(rest.sum()) > 0 else weights
        sums = torch.cumsum(weights, 0)
        token = int(torch.searchsorted(sums, u[b][K] * float(sums[-1]), right=True))
        n_acc.append(n)
        tokens.append(draft[b][:n] + [token] + [-1] * (K - n))
    return [torch.tensor(n_acc, dtype=torch.int32), torch.tensor(tokens, dtype=torch.int32)]


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------------

def work(case):
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "verify":
        # every sequence reads a row of p, and one of q where a draft fails (0.8 of them pass), and K pairs of probabilities
        drafts = case["K"] / 2 if case["ragged"] else case["K"]
        return {"bytes": case["B"] * (case["V"] * size * (2 - 0.8 ** drafts) + 2 * drafts * size + 12 * case["K"]),
                "flops": 2 * case["B"] * case["V"]}
    B, T, Hq, Hkv, D = (case[k] for k in ("B", "T", "Hq", "Hkv", "D"))
    if case["op"] == "append":
        rows = B * T / 2 if case["ragged"] else B * T
        return {"bytes": rows * (Hq + 2 * Hkv) * D * size * 2, "flops": rows * (Hq + Hkv) * case["R"] * 3}
    length = (case["least"] + case["most"]) / 2
    n = min(T, length)
    pairs = n * (length - (n - 1) / 2)  # (token, key it sees)
    return {"bytes": B * (2 * length * Hkv + 2 * n * Hq) * D * size, "flops": 4 * B * pairs * Hq * D}
