"""Trees of drafted tokens and the cache's budget in 64 bits (or whole numbers) on the CPU, one sequence, head
and token at a time, and how far a correct 32-bit computation may be from them."""

from __future__ import annotations

import math

import torch

from kv_reference import TINY, UNIT


def tree(parent, q_first, words):
    """(seen, depth): every token's chain of parents, walked."""
    n = parent.numel()
    seen, depth = torch.zeros(n, words, dtype=torch.int64), torch.zeros(n, dtype=torch.int32)
    for s in range(q_first.numel() - 1):
        t0, t1 = int(q_first[s]), int(q_first[s + 1])
        for i in range(t1 - t0):
            bits, j, steps = 0, i, -1
            while j >= 0:
                bits |= 1 << j
                steps += 1
                p = int(parent[t0 + j])
                j = p if 0 <= p < j else -1
            seen[t0 + i], depth[t0 + i] = pack(bits, words), steps
    return seen, depth


def pack(bits: int, words: int) -> torch.Tensor:
    part = [(bits >> (64 * w)) & ((1 << 64) - 1) for w in range(words)]
    return torch.tensor([x - (1 << 64) if x >> 63 else x for x in part], dtype=torch.int64)


def bit(row, j) -> bool:
    return j < 64 * row.numel() and bool(int(row[j // 64]) >> (j % 64) & 1)


def places(table_row, count, page):
    return [(int(table_row[j // page]), j % page) for j in range(count)]


def tree_attention(q, k_pages, v_pages, q_first, seen, own_pages, own_len, group_first=None, prefix_pages=None,
                   prefix_len=None, scale=None):
    """(out, lse, out bound, lse bound); the bounds are those of kv_reference.attention, whose terms are the
    same: one rounding of the output and of each exponential, 32-bit sums of d products, 2^-16 for
    exponentials, sums and rescalings."""
    dtype, d = q.dtype, q.shape[2]
    kp, vp, page, hkv = k_pages.double(), v_pages.double(), k_pages.shape[1], k_pages.shape[2]
    ratio, scale = q.shape[1] // hkv, d ** -0.5 if scale is None else scale
    out, out_tol = (torch.zeros(q.shape, dtype=torch.float64) for _ in range(2))
    lse, lse_tol = torch.full(q.shape[:2], -math.inf, dtype=torch.float64), torch.zeros(q.shape[:2], dtype=torch.float64)
    group = {}
    for g in range(0 if group_first is None else prefix_len.numel()):
        for s in range(int(group_first[g]), int(group_first[g + 1])):
            group[s] = g
    u = UNIT[dtype]
    for s in range(own_len.numel()):
        t0, t1, own = int(q_first[s]), int(q_first[s + 1]), int(own_len[s])
        first = own - (t1 - t0)
        shared = places(prefix_pages[group[s]], int(prefix_len[group[s]]), page) if s in group else []
        mine = places(own_pages[s], own, page)
        for t in range(t0, t1):
            at = shared + [p for j, p in enumerate(mine) if j < first or bit(seen[t], j - first)]
            at = [p for p in at if 0 <= p[0] < kp.shape[0]]
            if not at:
                continue
            at = torch.tensor(at).T
            k, v = kp[at[0], at[1]], vp[at[0], at[1]]
            x = q[t].double().view(hkv, ratio, d)
            score = torch.einsum("hrd,khd->hrk", x, k) * scale
            size = torch.einsum("hrd,khd->hrk", x.abs(), k.abs()).amax(-1) * abs(scale)
            e = (d + 4) * 2.0 ** -24 * size
            l = torch.logsumexp(score, -1)
            p = torch.exp(score - l[..., None])
            o, weight = torch.einsum("hrk,khd->hrd", p, v), torch.einsum("hrk,khd->hrd", p, v.abs())
            tol = u * o.abs() + (u + 2 * e[..., None] + 2.0 ** -16) * weight
            tol = tol + TINY[dtype] * (1 + v.abs().sum(0)[:, None])
            out[t], out_tol[t], lse[t] = o.reshape(-1, d), tol.reshape(-1, d), l.reshape(-1)
            lse_tol[t] = (e + 2.0 ** -18 * (1 + l.abs() + score.abs().amax(-1))).reshape(-1)
    return out, lse, out_tol, lse_tol


def accept(k_pages, v_pages, q_first, seen, leaf, own_pages, own_len):
    """(k_pages, v_pages, len_out) as they are to be."""
    kp, vp, page = k_pages.clone(), v_pages.clone(), k_pages.shape[1]
    length = own_len.clone()
    for s in range(own_len.numel()):
        n, own = int(q_first[s + 1]) - int(q_first[s]), int(own_len[s])
        mine, kept = places(own_pages[s], own, page), max(0, own - n)
        to = kept
        if 0 <= int(leaf[s]) < n:
            for j in range(n):
                if bit(seen[int(q_first[s]) + int(leaf[s])], j) and own - n + j >= 0:
                    (p, i), (x, y) = mine[own - n + j], mine[to]
                    if 0 <= p < kp.shape[0] and 0 <= x < kp.shape[0]:
                        kp[x, y], vp[x, y] = k_pages[p, i], v_pages[p, i]
                    to += 1
        length[s] = to
    return kp, vp, length


def weigh(q, k_pages, q_first, own_pages, own_len, lse, weights, born, positions, scale=None):
    """(weights, born, bound of the weights). The bound: a score's 32-bit sum of d products is off by
    (d + 4) 2^-24 of the sum of their sizes; the exponent's product with log2(e), its difference to the lse
    and the exponential itself by 2^-22 (1 + |score| + |lse|); each of the additions of a key's terms, one
    for each 16 rows and up to 12 more, by 2^-24 of the sum."""
    d, page, hkv = q.shape[2], k_pages.shape[1], k_pages.shape[2]
    ratio, scale = q.shape[1] // hkv, d ** -0.5 if scale is None else scale
    out, births = weights.double().clone(), born.clone()
    tol = torch.zeros_like(out)
    for s in range(own_len.numel()):
        t0, t1, own = int(q_first[s]), int(q_first[s + 1]), int(own_len[s])
        n = t1 - t0
        mine = places(own_pages[s], own, page)
        for j, (p, i) in enumerate(mine):
            if not 0 <= p < k_pages.shape[0]:
                continue
            new = j - (own - n)
            old = torch.zeros(hkv, dtype=torch.float64) if new >= 0 else weights[p, :, i].double()
            x = q[t0 + max(0, new):t1].double().view(-1, hkv, ratio, d)
            k = k_pages[p, i].double()
            score = torch.einsum("thrd,hd->thr", x, k) * scale
            size = torch.einsum("thrd,hd->thr", x.abs(), k.abs()) * abs(scale)
            l = lse[t0 + max(0, new):t1].double().view(-1, hkv, ratio)
            e = torch.exp(score - l)
            e = torch.where(l == math.inf, torch.zeros_like(e), e)
            rel = (d + 4) * 2.0 ** -24 * size + 2.0 ** -22 * (1 + score.abs() + torch.where(l.isfinite(), l.abs(), 0.0))
            out[p, :, i] = old + e.sum((0, 2))
            tol[p, :, i] = (2 * rel * e).sum((0, 2)) + (n * ratio / 16 + 12) * 2.0 ** -24 * out[p, :, i].abs() + 2.0 ** -120
            if new >= 0:
                births[p, :, i] = positions[t0 + new]
    return out, births, tol


def evict(k_pages, v_pages, own_pages, own_len, weights, born, total, keep, sinks=0, recent=0):
    """(k_pages, v_pages, weights, born, len_out) as they are to be, weights and born in place."""
    kp, vp, w, b = (x.clone() for x in (k_pages, v_pages, weights, born))
    page, pages = k_pages.shape[1], k_pages.shape[0]
    length = own_len.clone()
    for s in range(own_len.numel()):
        own = int(own_len[s])
        length[s] = min(own, keep)
        mine = places(own_pages[s], own, page)
        for h in range(k_pages.shape[2]):
            def rank(j):
                p, i = mine[j]
                if not 0 <= p < pages:
                    return (3, 0.0, j)
                x, at = float(weights[p, h, i]), int(born[p, h, i])
                if at < sinks or at >= int(total[s]) - recent:
                    return (0, 0.0, j)
                return (2, 0.0, j) if math.isnan(x) else (1, -x, j)
            kept = {j for _, _, j in sorted(rank(j) for j in range(own))[:keep]}
            free, moving = [j for j in range(min(keep, own)) if j not in kept], sorted(j for j in kept if j >= keep)
            assert len(free) == len(moving)
            for to, j in zip(free, moving):
                (x, y), (p, i) = mine[to], mine[j]
                if 0 <= x < pages and 0 <= p < pages:
                    kp[x, y, h], vp[x, y, h] = k_pages[p, i, h], v_pages[p, i, h]
                    w[x, h, y], b[x, h, y] = weights[p, h, i], born[p, h, i]
    return kp, vp, w, b, length
