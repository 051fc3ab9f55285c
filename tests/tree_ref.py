"""Definitions of the calls for rounds of drafted trees and windowed caches, in 64 bits on the host, and how far a result may be off."""
import math

import numpy as np
import torch

from round_ref import F32, HALF

ALL = 1 << 30


def random_tree(B, N, seed, reach=8, chain=False, roots=1):
    """Parents int32 [B, N], earlier nodes at most `reach` back; the first `roots` nodes have none."""
    g = torch.Generator().manual_seed(seed)
    n = torch.arange(N)
    up = n - 1 - (0 if chain else (torch.rand(B, N, generator=g) * n.clamp(max=reach)).long())
    return torch.where(n < roots, -1, up.expand(B, N)).to(torch.int32)


def lines(parents, n):
    """(depth of every node, whether node j is node i or one of its ancestors): entries that name no earlier node are none."""
    depth, line = [], torch.zeros(n, n, dtype=torch.bool)
    for t in range(n):
        up = int(parents[t])
        if 0 <= up < t:
            line[t] = line[up]
        line[t, t] = True
        depth.append(depth[up] + 1 if 0 <= up < t else 0)
    return torch.tensor(depth, dtype=torch.long), line


def sight(length, n, window=ALL, sinks=0, parents=None):
    """Which slots the last n of `length` tokens see (bool [n, max(length, 0)])."""
    held, slots = length - n, torch.arange(max(length, 0))
    if parents is None:
        place, of = held + torch.arange(n), slots
        sees = slots[None] <= place[:, None]
    else:
        depth, line = lines(parents, n)
        place, of = held + depth, slots.clone()
        sees = (slots[None] < held).expand(n, -1).clone()
        nodes = slots >= held
        of[nodes] = held + depth[(slots - held)[nodes]]
        sees[:, nodes] = line[:, (slots - held)[nodes]]
    sees = sees & ((of[None] > place[:, None] - window) | (of[None] < sinks))
    return sees & (held + torch.arange(n) >= 0)[:, None]


def attention(q, k_pool, v_pool, table, lens, n_new=None, scale=None, window=ALL, sinks=0, parents=None):
    """As round_ref.attention, with which keys a token sees; parents: [B, T] or [T]."""
    q, kp, vp, table, lens = q.cpu(), k_pool.cpu(), v_pool.cpu(), table.cpu(), lens.cpu().tolist()
    B, T, Hq, D = q.shape
    n_pages, page, Hkv, _ = kp.shape
    G, cols = Hq // Hkv, table.shape[1]
    scale = 1 / math.sqrt(D) if scale is None else scale
    half = HALF[q.dtype]
    out, lse, tol = torch.zeros(B, T, Hq, D, dtype=torch.float64), torch.full((B, T, Hq), -math.inf, dtype=torch.float64), torch.zeros(B, T, Hq, D, dtype=torch.float64)
    ltol, there = torch.zeros(B, T, Hq, dtype=torch.float64), torch.zeros(B, T, dtype=torch.bool)
    if parents is not None:
        parents = parents.cpu().expand(B, T)
    for b in range(B):
        n = T if n_new is None else min(max(int(n_new[b]), 0), T)
        there[b, :n] = True
        if not n or lens[b] <= 0:
            continue
        sees = sight(lens[b], n, window, sinks, None if parents is None else parents[b])
        slots = torch.tensor([j for j in sees.any(0).nonzero()[:, 0].tolist() if j < cols * page and 0 <= int(table[b, j // page]) < n_pages], dtype=torch.long)
        if not len(slots):
            continue
        keys = kp[table[b, slots // page].long(), slots % page].double()
        vals = vp[table[b, slots // page].long(), slots % page].double()
        for t in range(n):
            mine = sees[t, slots]
            m = int(mine.sum())
            if not m:
                continue
            k = keys[mine].repeat_interleave(G, 1).transpose(0, 1)                  # [Hq, m, D]
            v = vals[mine].repeat_interleave(G, 1).transpose(0, 1)
            x = q[b, t].double()
            s = (k @ x[:, :, None])[..., 0] * scale                                 # [Hq, m]
            top = s.amax(1)
            ok = top > -math.inf
            w = torch.where(ok[:, None], torch.exp(s - torch.where(ok, top, 0.0)[:, None]), 0.0)
            total = w.sum(1)
            lse[b, t] = torch.where(ok, top + torch.log(torch.where(ok, total, 1.0)), -math.inf)
            w = w / torch.where(ok, total, 1.0)[:, None]
            out[b, t] = (w[:, None] @ v)[:, 0]
            # (the bound of round_ref.attention: scores, weights, their sum, the roundings to bf16, for m keys)
            d = ((D + 8) * F32 * (k.abs() @ x.abs()[:, :, None])[..., 0] * abs(scale) + 4 * F32 * s.abs()).amax(1)
            rel = 2 * d + 4 * F32 + (m + 40) * F32
            rounded = half if q.dtype == torch.bfloat16 else 0.0
            mass = (w[:, None] @ v.abs())[:, 0]
            tol[b, t] = torch.where(ok[:, None], (mass + out[b, t].abs()) * (rel + rounded)[:, None] * 1.05 + half * out[b, t].abs(), 0.0)
            ltol[b, t] = torch.where(ok, rel + rounded + 4 * F32 * torch.where(ok, lse[b, t], 0.0).abs(), 0.0)
    return out, lse, tol, ltol, there


def scores(logits, tokens, top, temperature=1.0, n_new=None):
    """(logprobs, entropy, top_ids, top_logprobs) and how far the three numbers may be off, for rows of finite logits and -inf."""
    x = logits.double().cpu().numpy()
    B, T, V = x.shape
    temperature = float(np.float32(temperature))
    lp, ent = np.zeros((B, T)), np.zeros((B, T))
    ids, alt = np.full((B, T, top), -1, np.int64), np.zeros((B, T, top))
    lp_tol, ent_tol, alt_tol = np.zeros((B, T)), np.zeros((B, T)), np.zeros((B, T, top))
    for b in range(B):
        for t in range(T if n_new is None else min(max(int(n_new[b]), 0), T)):
            row = x[b, t]
            m = row.max()
            alt[b, t] = -np.inf
            token = None if tokens is None else int(tokens[b, t])
            if m == -np.inf:
                lp[b, t] = -np.inf
                continue
            d = (row - m) / temperature
            with np.errstate(over="ignore"):
                w = np.exp(d)
            total = w.sum()
            p, ln = w / total, math.log(total)
            far = np.where(p > 0, -d, 0.0)
            # An exponent takes three roundings (difference, factor, its product), its power one of 2^-23; sums round once a term of a lane (V / 256, fewer where
            # workgroups share a row) and, for the factors of larger maxima, four times every 32, then some 60 times between lanes and wavefronts.
            adds = V / 256 + V / 2048 + 60
            rel = F32 * (3 * float((p * far).sum()) + 2 + adds)
            ent[b, t] = ln + float((p * far).sum())
            ent_tol[b, t] = rel + F32 * (4 * abs(ln) + (3 * float((p * far * far).sum()) + (6 + 2 * adds) * float((p * far).sum())) + 2 * rel) + 2 * rel * float((p * far).sum()) + F32
            of = lambda v: (4 * abs(v) + 2 * abs(ln) + abs(v - ln)) * F32 + rel + F32
            if token is not None:
                lp[b, t] = d[token] - ln if 0 <= token < V else -np.inf
                lp_tol[b, t] = of(d[token]) if 0 <= token < V and np.isfinite(d[token]) else 0.0
            order = np.argsort(-row, kind="stable")[:top]
            order = order[row[order] > -np.inf]
            ids[b, t, : len(order)], alt[b, t, : len(order)] = order, d[order] - ln
            alt_tol[b, t, : len(order)] = [of(v) for v in d[order]]
    # (what is below the least number of 32 bits rounds to -inf there)
    lp[lp < -np.finfo(np.float32).max], alt[alt < -np.finfo(np.float32).max] = -np.inf, -np.inf
    return (lp, ent, ids, alt), (lp_tol, ent_tol, alt_tol)


def check_scores(got, want, tol, tokens=True):
    lp, ent, ids, alt = want
    near = lambda a, b, t: np.all((a == b) | (np.abs(a - b) <= t))
    with np.errstate(invalid="ignore"):
        if tokens:
            assert near(got["logprobs"].double().cpu().numpy(), lp, tol[0])
        else:
            assert got["logprobs"] is None
        assert near(got["entropy"].double().cpu().numpy(), ent, tol[1]), np.abs(got["entropy"].double().cpu().numpy() - ent).max()
        if ids.shape[2]:
            assert np.array_equal(got["top_ids"].cpu().numpy(), ids)
            assert near(got["top_logprobs"].double().cpu().numpy(), alt, tol[2])
        else:
            assert got["top_ids"] is None and got["top_logprobs"] is None


def walked(tokens, parents, p=None, u=None, choices=None, n_new=None):
    """(n_acc, tokens, path) by the definition."""
    tokens, (B, N) = tokens.cpu().tolist(), tokens.shape
    parents = parents.cpu().expand(B, N).tolist()
    p = None if p is None else p.double().cpu().numpy()
    u = None if u is None else u.double().cpu().numpy()
    counts, out, paths = [], [], []
    for b in range(B):
        n = N if n_new is None else min(max(int(n_new[b]), 0), N)
        drawn, path, at = [], [], 0 if n else -1
        while at >= 0:
            path.append(at)
            if choices is not None:
                y = int(choices[b, at])
            else:
                w = np.where(np.isfinite(p[b, at]) & (p[b, at] > 0), p[b, at], 0.0)
                sums, heavy = np.cumsum(w), np.flatnonzero(w > 0)
                over = heavy[sums[heavy] > u[b, len(drawn)] * sums[-1]] if len(heavy) else heavy
                y = -1 if not len(heavy) else int(over[0]) if len(over) else int(heavy[-1])
            drawn.append(y)
            at = next((c for c in range(at + 1, n) if parents[b][c] == at and tokens[b][c] == y and y >= 0), -1)
        counts.append(len(path) - 1)
        out.append(drawn + [-1] * (N - len(drawn)))
        paths.append(path + [-1] * (N - len(path)))
    return counts, out, paths


def kept(pool, table, held, path, page):
    """A pool [..., pages, page, heads, dim] on the host after the path's rows moved together."""
    old, new = pool.clone(), pool.clone()
    n_pages, cols = pool.shape[-4], table.shape[1]

    def row(b, slot):
        if slot < 0 or slot // page >= cols or not 0 <= int(table[b, slot // page]) < n_pages:
            return None
        return int(table[b, slot // page]), slot % page

    for b in range(path.shape[0]):
        before = -1
        if int(held[b]) < 0:
            continue
        for i, n in enumerate(path[b].tolist()):
            if n <= before or n >= path.shape[1]:
                break
            before = n
            x, y = row(b, int(held[b]) + n), row(b, int(held[b]) + i)
            if x is not None and y is not None:
                new[..., y[0], y[1], :, :] = old[..., x[0], x[1], :, :]
    return new
