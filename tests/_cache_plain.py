"""The 4-bit cache's records, attention over them and eviction, plainly and in 64 bits."""
import math

import torch

CODES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
SCALES = [(b & 7) * 2.0 ** -9 if b < 8 else (8 + (b & 7)) * 2.0 ** ((b >> 3) - 10) for b in range(127)] + \
         [math.nan]


def nearest(x, values):
    """The index of the nearest of ascending values to each x >= 0 (64 bits), ties to the even index."""
    v = torch.tensor(values, dtype=torch.float64, device=x.device)
    hi = torch.bucketize(x, v).clamp(1, len(values) - 1)       # v[hi - 1] < x <= v[hi], or x outside
    below, above = x - v[hi - 1], v[hi] - x
    up = (above < below) | ((above == below) & (hi % 2 == 0))
    return torch.where(up, hi, hi - 1)


def round_values(x, unit=1.0):
    """What the cache keeps of x [..., d], in 64 bits."""
    g = x.double().unflatten(-1, (-1, 16)) / unit
    top = g.abs().amax(-1)
    table = torch.tensor(SCALES, dtype=torch.float64, device=x.device)
    s = table[nearest(top.clamp(max=1e300) / 6, SCALES[:127]).clamp(min=1)]
    code = nearest((g.abs() / s[..., None]).nan_to_num(0.0, posinf=9.0), CODES)
    v = torch.tensor(CODES, dtype=torch.float64, device=x.device)[code]
    v = torch.where(torch.signbit(g), -v, v) * s[..., None]
    return (torch.where(top.isnan()[..., None], math.nan, v) * unit).flatten(-2)


def values(half, unit=1.0):
    """Half records (codes, then eight scales) [..., d / 2 + 8] as 64-bit values."""
    d = 2 * (half.shape[-1] - 8)
    b = half[..., :d // 2].long()
    c = torch.stack([b & 15, b >> 4], -1).flatten(-2)
    v = torch.tensor(CODES + [-x for x in CODES], dtype=torch.float64, device=half.device)[c]
    s = torch.tensor(SCALES + SCALES, dtype=torch.float64, device=half.device)[
        half[..., d // 2:d // 2 + d // 16].long()]
    return (v.unflatten(-1, (-1, 16)) * s[..., None]).flatten(-2) * unit


def attention(q, cache, lens, scale, k_unit=1.0, v_unit=1.0):
    """(out, lse, what each position gets, sum of p |v|) in 64 bits; NaN where there is no sequence."""
    N, T, Hq, d = q.shape
    S, H, half = cache.shape[1], cache.shape[2], d // 2 + 8
    rep = Hq // H
    out = torch.full(q.shape, math.nan, dtype=torch.float64, device=q.device)
    A, lse = out.clone(), out[..., 0].clone()
    w = torch.zeros((N, H, S), dtype=torch.float64, device=q.device)
    for n in range(N):
        if int(lens[n]) < 0:
            continue
        L = min(int(lens[n]), S)
        kk = values(cache[n, :L, :, :half], k_unit)
        vv = values(cache[n, :L, :, half:], v_unit)
        for t in range(T):
            m = max(L - (T - 1 - t), 0)
            s = torch.einsum("hrd,jhd->hrj", q[n, t].double().view(H, rep, d), kk[:m]) * scale
            lse[n, t] = torch.logsumexp(s, 2).view(-1) if m else -math.inf
            p = torch.softmax(s, 2)
            out[n, t] = torch.einsum("hrj,jhd->hrd", p, vv[:m]).reshape(Hq, d)
            A[n, t] = torch.einsum("hrj,jhd->hrd", p, vv[:m].abs()).reshape(Hq, d)
            there = p.isfinite().all(2)[:, :, None]
            w[n, :, :m] += torch.where(there, p, 0.0).sum(1)
    return out, lse, w, A


def evict(weights, lens, budget, recent, first):
    """(kept, new lengths) of weights [N, H, S]: lists of the positions that stay."""
    N, H, S = weights.shape
    kept = torch.full((N, H, budget), -1, dtype=torch.int32)
    new = []
    for n in range(N):
        raw = int(lens[n])
        L = min(max(raw, 0), S)
        new.append(raw if raw < 0 else min(L, budget))
        for h in range(H):
            w = weights[n, h, :L].tolist()
            if L <= budget:
                stay = list(range(L))
            else:
                stay = list(range(first)) + list(range(L - recent, L))
                rest = sorted(range(first, L - recent),
                              key=lambda j: (w[j] != w[j], -w[j] if w[j] == w[j] else 0.0, j))
                stay = sorted(stay + rest[:budget - first - recent])
            kept[n, h, :len(stay)] = torch.tensor(stay, dtype=torch.int32)
    return kept, torch.tensor(new, dtype=torch.int32)
