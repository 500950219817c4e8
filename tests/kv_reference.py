"""The paged key/value cache's operators in 64 bits on the CPU, one sequence and head at a time,
and how far a correct 32-bit computation with one rounding to 16 bits may be from them."""

from __future__ import annotations

import math

import torch

# half the spacing of a type's values relative to them, and of its smallest ones
UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.float16, torch.bfloat16)}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def angles(positions, rot_dim, base=10000.0, factor=1.0, original=0, slow=1.0, fast=32.0):
    out = torch.zeros(positions, rot_dim // 2, dtype=torch.float64)
    for i in range(rot_dim // 2):
        f = base ** (-2 * i / rot_dim)
        keep = min(max((original * f / (2 * math.pi) - slow) / (fast - slow), 0.0), 1.0) if original else 0.0
        out[:, i] = torch.arange(positions, dtype=torch.float64) * (f * (keep + (1 - keep) / factor))
    return out


def heads(x, weight, eps, table, positions, interleaved):
    """(value, bound) of heads [tokens, heads, d] normed and rotated; table float32 as the call
    gets it. The bound: one rounding to the type of x, and 32-bit arithmetic: about twenty
    roundings of 2^-24 relative to the terms of each sum, taken as 2^-18."""
    dtype, x = x.dtype, x.double()
    if weight is not None:
        x = x * weight.double() / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt()
    size = x.abs()
    if table is not None:
        row = table.double()[positions.long()][:, None]
        h = table.shape[1] // 2
        c, s = row[..., :h], row[..., h:]
        a, b = (slice(0, 2 * h, 2), slice(1, 2 * h, 2)) if interleaved else (slice(0, h), slice(h, 2 * h))
        y, t = x.clone(), size.clone()
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        t[..., a] = size[..., a] * c.abs() + size[..., b] * s.abs()
        t[..., b] = size[..., b] * c.abs() + size[..., a] * s.abs()
        x, size = y, t
    return x, UNIT[dtype] * x.abs() + 2.0 ** -18 * size + TINY[dtype]


def attention(q, k_pages, v_pages, q_first, own_pages, own_len, group_first=None, prefix_pages=None, prefix_len=None,
              scale=None):
    """(out, lse, out bound, lse bound), everything on the CPU. Only what a row sees is read.

    The bounds, u the type's unit: out is rounded once (u |out|); each exp(score - max) is
    rounded to the type (u sum p |v|, and where that type's smallest values end, their half
    spacing); a score's 32-bit sum of d products is off by at most (d + 4) 2^-24 of the sum of
    their sizes, e, which changes its p by the factor exp(+-2 e) with the sum's; 2^-16 of
    sum p |v| is for the 32-bit exponentials, sums and rescalings of up to 2^7 pieces."""
    dtype, d = q.dtype, q.shape[2]
    q, kp, vp = q.double(), k_pages.double(), v_pages.double()
    page, hkv = kp.shape[1], kp.shape[2]
    ratio = q.shape[1] // hkv
    scale = d ** -0.5 if scale is None else scale
    out = torch.zeros(q.shape, dtype=torch.float64)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    out_tol, lse_tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape[:2], dtype=torch.float64)
    group = {}
    for g in range(0 if group_first is None else prefix_len.numel()):
        for s in range(int(group_first[g]), int(group_first[g + 1])):
            group[s] = g

    def places(table_row, count):
        return [(int(table_row[j // page]), j % page) for j in range(count)]

    for s in range(own_len.numel()):
        t0, t1 = int(q_first[s]), int(q_first[s + 1])
        n, own = t1 - t0, int(own_len[s])
        shared = places(prefix_pages[group[s]], int(prefix_len[group[s]])) if s in group else []
        mine = places(own_pages[s], own)
        for i in range(n):
            seen = shared + mine[:max(0, own - n + i + 1)]
            seen = [(p, o) for p, o in seen if 0 <= p < kp.shape[0]]
            if not seen:
                continue
            at = torch.tensor([p for p, _ in seen]), torch.tensor([o for _, o in seen])
            k, v = kp[at], vp[at]  # [keys, hkv, d]
            x = q[t0 + i].view(hkv, ratio, d)
            score = torch.einsum("hrd,khd->hrk", x, k) * scale
            size = torch.einsum("hrd,khd->hrk", x.abs(), k.abs()).amax(-1) * abs(scale)
            e = (d + 4) * 2.0 ** -24 * size  # [hkv, ratio]
            l = torch.logsumexp(score, -1)
            p = torch.exp(score - l[..., None])
            o = torch.einsum("hrk,khd->hrd", p, v)
            weight = torch.einsum("hrk,khd->hrd", p, v.abs())
            u = UNIT[dtype]
            tol = u * o.abs() + (u + 2 * e[..., None] + 2.0 ** -16) * weight
            tol = tol + TINY[dtype] * (1 + v.abs().sum(0)[:, None])
            out[t0 + i], out_tol[t0 + i] = o.reshape(-1, d), tol.reshape(-1, d)
            lse[t0 + i] = l.reshape(-1)
            lse_tol[t0 + i] = (e + 2.0 ** -18 * (1 + l.abs() + score.abs().amax(-1))).reshape(-1)
    return out, lse, out_tol, lse_tol


def near(got, want, tol, what):
    got = got.detach().cpu().double()
    fine = torch.isfinite(want)
    same = (torch.isnan(got) == torch.isnan(want)) & (fine == torch.isfinite(got))
    same &= fine | torch.isnan(want) | (got == want)
    assert bool(same.all()), f"{what}: {int((~same).sum())} values are not finite where they should be, or the reverse"
    off = (got - want).abs()[fine]
    bad = off > tol[fine]
    assert not bool(bad.any()), (f"{what}: {int(bad.sum())} of {bad.numel()} off by more than their bound, "
                                 f"worst {float((off / tol[fine].clamp(min=1e-300)).max()):.2f} of it")
