"""Definitions of the calls for a round of the caller's own models, in 64 bits on the host, and how far a result may be off."""
import math

import numpy as np
import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}       # half a step, relative to the value
F32 = 2.0 ** -24


def paged(B, cols, page, H, D, dtype, seed, order="token", spare=0, fill=None):
    """Pools (logical shape [pages, page, H, D]) and a page table in no order; `order`: how they lie in memory."""
    g = torch.Generator().manual_seed(seed)
    n = B * cols + spare
    lie = {"token": (0, 1, 2, 3), "head": (0, 2, 1, 3)}[order]
    back = [lie.index(i) for i in range(4)]
    make = lambda: (torch.randn(n, page, H, D, generator=g) if fill is None else torch.full((n, page, H, D), fill)).to(dtype)
    pools = [make().permute(lie).contiguous().cuda().permute(back) for _ in range(2)]
    return pools[0], pools[1], torch.randperm(n, generator=g)[: B * cols].to(torch.int32).view(B, cols).cuda()


def attention(q, k_pool, v_pool, table, lens, n_new=None, scale=None):
    """(out, lse, how far off out may be, how far off lse may be, rows that are there), float64 on the host."""
    q, kp, vp, table, lens = q.cpu(), k_pool.cpu(), v_pool.cpu(), table.cpu(), lens.cpu().tolist()
    B, T, Hq, D = q.shape
    n_pages, page, Hkv, _ = kp.shape
    G, cols = Hq // Hkv, table.shape[1]
    scale = 1 / math.sqrt(D) if scale is None else scale
    half = HALF[q.dtype]
    out, lse, tol = torch.zeros(B, T, Hq, D, dtype=torch.float64), torch.full((B, T, Hq), -math.inf, dtype=torch.float64), torch.zeros(B, T, Hq, D, dtype=torch.float64)
    ltol, there = torch.zeros(B, T, Hq, dtype=torch.float64), torch.zeros(B, T, dtype=torch.bool)
    for b in range(B):
        n = T if n_new is None else min(max(int(n_new[b]), 0), T)
        length = max(lens[b], 0)
        slots = [j for j in range(min(length, cols * page)) if 0 <= int(table[b, j // page]) < n_pages]
        at = torch.tensor(slots, dtype=torch.long)
        keys = kp[table[b, at // page].long(), at % page].double()      # [n, Hkv, D]
        vals = vp[table[b, at // page].long(), at % page].double()
        for t in range(n):
            there[b, t] = True
            m = int((at < length - n + t + 1).sum())
            if not m:
                continue
            for h in range(Hq):
                k, v, x = keys[:m, h // G], vals[:m, h // G], q[b, t, h].double()
                s = k @ x * scale
                top = s.max()
                if top == -math.inf:
                    continue
                w = torch.exp(s - top)
                lse[b, t, h] = top + torch.log(w.sum())
                w = w / w.sum()
                out[b, t, h] = w @ v
                # A score: D products summed in fp32 (each partial sum rounds), the factor and the maximum's subtraction; base 2 scores
                # are 1.44 times as large.  A weight is off by twice that (its own and the maximum's), 2^-22 for exp2 itself, and by the
                # rounding to the values' type (bf16); the normaliser by as much again.  Sums over m keys round m times.
                d = float(((D + 8) * F32 * (k.abs() @ x.abs()) * abs(scale) + 4 * F32 * s.abs()).max())
                rel = 2 * d + 4 * F32 + (m + 40) * F32
                mass = w @ v.abs()
                tol[b, t, h] = (mass + out[b, t, h].abs()) * (rel + (half if q.dtype == torch.bfloat16 else 0.0)) * 1.05 + half * out[b, t, h].abs()
                ltol[b, t, h] = rel + (half if q.dtype == torch.bfloat16 else 0.0) + 4 * F32 * abs(float(lse[b, t, h]))
    return out, lse, tol, ltol, there


def check_attention(got, lse, ref, before=None):
    out, want_lse, tol, ltol, there = ref
    got = got.double().cpu()
    assert torch.isfinite(got[there]).all()
    off = (got - out).abs()
    assert bool((off[there] <= tol[there]).all()), float((off / tol.clamp(min=1e-300))[there].max())
    if lse is not None:
        a, b = lse.double().cpu()[there], want_lse[there]
        assert torch.equal(a == -math.inf, b == -math.inf)
        ok = b > -math.inf
        assert bool(((a - b).abs()[ok] <= ltol[there][ok]).all()), float(((a - b).abs()[ok] / ltol[there][ok]).max())
    if before is not None:
        assert torch.equal(got[~there], before.double().cpu()[~there])


def rotated(x, positions, freq, interleaved, amplitude):
    """(turned heads, how far off they may be) in 64 bits; x: [B, T, H, D], positions [B, T]."""
    half = HALF[x.dtype]
    x, f = x.double().cpu(), torch.as_tensor(freq).double().cpu()
    R = 2 * f.numel()
    ang = positions.double().cpu()[:, :, None, None] * f
    c, s = amplitude * ang.cos(), amplitude * ang.sin()
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., : R // 2], x[..., R // 2:R])
    ya, yb = a * c - b * s, a * s + b * c
    # the angle's rest of a turn in fp32 (2^-26 turns: 1.6 * 2^-24 rad), sine and cosine (2 units of 2^-24 relative to 1 each way), the
    # amplitude, a product and the sum: under 8 * 2^-24 of what goes in
    # and both sides' angles are 64-bit products, off by 2^-53 of themselves a rounding
    t = (8 * F32 + 4 * 2.0 ** -53 * ang.abs()) * abs(amplitude) * (a.abs() + b.abs())
    y, tol = x.clone(), torch.zeros_like(x)
    ia, ib = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    y[..., ia], y[..., ib] = ya, yb
    tol[..., ia], tol[..., ib] = t + half * ya.abs() * (1 + 2 ** -7) + half * t, t + half * yb.abs() * (1 + 2 ** -7) + half * t
    return y, tol


def verified(draft, q, p, u, n_draft=None):
    """(n_acc, tokens) by the definition."""
    draft, p, u = draft.cpu().tolist(), p.double().cpu().numpy(), u.double().cpu().numpy()
    q = None if q is None else q.double().cpu().numpy()
    B, K, V = len(draft), len(draft[0]), p.shape[2]
    counts, tokens = [], []
    for b in range(B):
        k = K if n_draft is None else min(max(int(n_draft[b]), 0), K)
        n = 0
        while n < k:
            x = draft[b][n]
            if not (0 <= x < V) or not (u[b, n] * (1.0 if q is None else q[b, n, x]) < p[b, n, x]):
                break
            n += 1
        base = np.where(np.isfinite(p[b, n]) & (p[b, n] > 0), p[b, n], 0.0)
        w = base
        if n < k:
            if q is None:
                w = base.copy()
                if 0 <= draft[b][n] < V:
                    w[draft[b][n]] = 0
            else:
                with np.errstate(invalid="ignore"):
                    w = p[b, n] - q[b, n]
                w = np.where(np.isfinite(w) & (w > 0), w, 0.0)
            if not w.sum() > 0:
                w = base
        sums, heavy = np.cumsum(w), np.flatnonzero(w > 0)
        token = -1
        if len(heavy):
            over = heavy[sums[heavy] > u[b, K] * sums[-1]]
            token = int(over[0]) if len(over) else int(heavy[-1])
        counts.append(n)
        tokens.append(draft[b][:n] + [token] + [-1] * (K - n))
    return counts, tokens
