"""The operators of the paged key/value cache, in their plain form and as the library's calls.

A case is a dict of plain values; its "op" names the operator of one pass:

  append   keys and values of new tokens go into a paged cache, rotated by their positions on
           the way, queries rotated in the same pass, each head normed first where "norm" is
           true: kv_append()
  attend   attention of a ragged batch over that cache, in which the sequences of a group share
           a prefix: prefix_attention()

A case fixes how many of everything there are: lengths are drawn from its "ragged" number, so
that the work of a pass does not depend on the seed. The seed draws the contents: keys, values,
queries, which pages of the cache hold them, and in which order. Head counts, widths and fp16
are the 7B decoder's of workloads/ (32 heads of 128), or of decoders whose heads share keys.
"""

import math
import random

import torch

own = False
DEVICE = "cuda"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _append(name, t, hq, hkv, d, rot, page, dtype, interleaved=False, norm=False, positions=4096, factor=1.0,
            skip=0.0, fused=True):
    return {"name": name, "op": "append", "t": t, "hq": hq, "hkv": hkv, "d": d, "rot": rot, "page": page,
            "dtype": dtype, "interleaved": interleaved, "norm": norm, "positions": positions, "factor": factor,
            "skip": skip, "fused": fused}


def _attend(name, b, nq, own_lo, own_hi, groups, prefix_lo, prefix_hi, hq, hkv, d, page, dtype, ragged, whole=False):
    """nq: most new tokens of a sequence (1 to nq are drawn); whole: nq of each, all of its own keys."""
    return {"name": name, "op": "attend", "b": b, "nq": nq, "own_lo": own_lo, "own_hi": own_hi, "groups": groups,
            "prefix_lo": prefix_lo, "prefix_hi": prefix_hi, "hq": hq, "hkv": hkv, "d": d, "page": page,
            "dtype": dtype, "ragged": ragged, "whole": whole}


def listed():
    return [
        # One user's next token in the 7B decoder: the smallest call, bound by latency.
        _append("append_one", 1, 32, 32, 128, 128, 16, "fp16", fused=False),
        # The next tokens of a full serving batch, heads normed, eight key heads.
        _append("append_decode_256", 256, 32, 8, 128, 128, 64, "bf16", norm=True, positions=32768, factor=4.0),
        # An odd count of prompt tokens, some of them padding, a model that rotates neighbouring
        # dimensions and half of each head only.
        _append("append_odd_1021", 1021, 28, 4, 64, 32, 16, "fp16", interleaved=True, skip=0.05),
        # A large chunk of long prompts: bound by memory.
        _append("append_prompt_16k", 16384, 32, 8, 128, 128, 64, "bf16", norm=True, positions=131072, factor=32.0),
        # One user, a short history, nothing shared: the smallest call.
        _attend("decode_one", 1, 1, 37, 37, 0, 0, 0, 32, 32, 128, 16, "fp16", 1),
        # A batch of chats behind one system prompt.
        _attend("decode_64_shared_2000", 64, 1, 1, 300, 1, 2000, 2000, 32, 8, 128, 64, "bf16", 2),
        # Several assistants with prompts of their own, small heads, an odd sharing of key heads.
        _attend("decode_192_groups", 192, 1, 1, 1000, 12, 16, 4096, 28, 4, 64, 16, "fp16", 3),
        # Many questions about one long document.
        _attend("decode_128_shared_8192", 128, 1, 1, 1024, 1, 8192, 8192, 32, 8, 128, 64, "bf16", 4),
        # One user with a very long history: few rows, a long axis.
        _attend("decode_long_131071", 1, 1, 131071, 131071, 0, 0, 0, 32, 8, 128, 64, "bf16", 5),
        # A few proposed tokens of each sequence checked at once; some sequences have fewer keys
        # than tokens, so that their first rows see nothing but the prefix, or nothing at all.
        _attend("verify_32x5", 32, 5, 1, 400, 2, 0, 1024, 32, 4, 128, 32, "bf16", 6),
        # Chunks of prompts of different lengths behind a shared prefix.
        _attend("extend_6x700", 6, 700, 700, 1500, 1, 4096, 4096, 32, 8, 128, 64, "bf16", 7),
        # A whole prompt of the 7B decoder, nothing shared: bound by the matrix units.
        _attend("prompt_8192", 1, 8192, 8192, 8192, 0, 0, 0, 32, 32, 128, 64, "fp16", 8, whole=True),
    ]


def _log(rng, lo, hi):
    return lo if hi <= lo else min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    d = rng.choice([64, 128, 128, 256])
    hkv = rng.choice([1, 2, 4, 5, 8, 8, 16, 32])
    hq = hkv * rng.choice([r for r in (1, 2, 3, 4, 4, 7, 8) if r * hkv <= 64])
    page, dtype = rng.choice([16, 32, 64, 128]), rng.choice(["fp16", "bf16"])
    if rng.random() < 0.35:
        norm, part = rng.random() < 0.5, rng.choice([1, 1, 2])
        c = _append("", _log(rng, 1, 16384), hq, hkv, d, d // part, page, dtype, rng.random() < 0.4, norm,
                    rng.choice([4096, 32768, 131072]), rng.choice([1.0, 4.0, 32.0]), rng.choice([0.0, 0.1]),
                    rng.random() < 0.7)
        while c["t"] * (hq + 2 * hkv) * d > 16384 * 48 * 128:
            c["t"] = 1 + c["t"] // 2
    else:
        kind = rng.choice(["one", "decode", "decode", "verify", "extend", "prompt"])
        groups = rng.choice([0, 1, 1, 3, 8])
        b, nq, lo, hi = 1, 1, 1, 65536
        if kind in ("decode", "verify"):
            b, hi = _log(rng, 2, 256), _log(rng, 1, 2048)
            nq = rng.randint(2, 9) if kind == "verify" else 1
        elif kind == "extend":
            b, nq = _log(rng, 1, 12), _log(rng, 16, 700)
            lo, hi = nq, nq + _log(rng, 1, 1500)
        elif kind == "prompt":
            nq = _log(rng, 16, 6000)
            lo = hi = nq
        if kind == "one":
            lo = hi = _log(rng, 1, hi)
        groups = min(groups, b)
        p = _log(rng, 1, 4096) if groups else 0
        # what the plain form gathers and scores stays below the largest listed cases'
        while hq * b * nq * (hi + p) > 1 << 31 or b * (hi + p) * hkv * d > 1 << 30:
            b, p, groups = max(1, b // 2), p // 2, min(groups, max(1, b // 2))
            if b == 1:
                nq = max(1, nq // 2)
                lo, hi = (nq, nq) if kind == "prompt" else (min(lo, max(1, hi // 2)), max(1, hi // 2))
                lo = min(lo, hi)
        c = _attend("", b, nq, lo, hi, groups, p // 2, p, hq, hkv, d, page, dtype, rng.randrange(1 << 20),
                    kind == "prompt")
    del c["name"]
    return c


def _lengths(case):
    """New tokens and own keys of each sequence, the first sequence of each group, the prefixes' lengths."""
    rng = random.Random(case["ragged"])
    b, g = case["b"], case["groups"]
    nq = [case["nq"] if case["whole"] or case["nq"] == 1 else rng.randint(1, case["nq"]) for _ in range(b)]
    keys = [_log(rng, case["own_lo"], case["own_hi"]) for _ in range(b)]
    first = [0] + sorted(rng.sample(range(1, b), g - 1)) + [b] if g else [0]
    prefix = [_log(rng, max(1, case["prefix_lo"]), case["prefix_hi"]) for _ in range(g)]
    if g and not case["prefix_lo"]:
        prefix[0] = 0  # a group that shares nothing
    return nq, keys, first, prefix


def _angles(case, dtype):
    """Rotation angles of every position [positions, rot / 2], the slow ones stretched by "factor"."""
    r, length = case["rot"], case["positions"] / case["factor"]
    theta = 10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64, device=DEVICE) / r)
    keep = ((length * theta / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
    theta = theta * (keep + (1.0 - keep) / case["factor"])
    return (torch.arange(case["positions"], dtype=torch.float64, device=DEVICE)[:, None] * theta[None]).to(dtype)


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEVICE)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEVICE)


def _page_table(per_row, order, at):
    """One row of page numbers for each count, filled up with -1; `order`: the cache's pages, shuffled."""
    width = max([1] + per_row)
    table = torch.full((len(per_row), width), -1, dtype=torch.int32, device=DEVICE)
    count = _ints(per_row)
    held = torch.arange(width, device=DEVICE)[None] < count[:, None]
    n = sum(per_row)
    table[held] = order[at:at + n].to(torch.int32)
    return table, at + n


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    dtype, hq, hkv, d, page = TYPES[case["dtype"]], case["hq"], case["hkv"], case["d"], case["page"]
    if case["op"] == "append":
        t = case["t"]
        if case["fused"]:  # one product gives queries, keys and values side by side
            rows = _randn(gen, t, (hq + 2 * hkv) * d).to(dtype).view(t, hq + 2 * hkv, d)
            q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
        else:
            q, k, v = (_randn(gen, t, h, d).to(dtype) for h in (hq, hkv, hkv))
        pages = -(-t // page) + 4
        slots = torch.randperm(pages * page, generator=gen, device=DEVICE)[:t]
        if case["t"] >= 1024:  # prompts fill whole pages, in any order
            order = torch.randperm(pages, generator=gen, device=DEVICE)
            i = torch.arange(t, device=DEVICE)
            slots = order[i // page] * page + i % page
        slots[torch.rand(t, generator=gen, device=DEVICE) < case["skip"]] = -1
        angles = _angles(case, torch.float64)
        s = {"op": "append", "q": q, "k": k, "v": v, "slots": slots, "interleaved": case["interleaved"],
             "k_pages": _randn(gen, pages, hkv, page, d).to(dtype).transpose(1, 2),
             "v_pages": _randn(gen, pages, hkv, page, d).to(dtype).transpose(1, 2),
             "positions": torch.randint(0, case["positions"], (t,), generator=gen, device=DEVICE, dtype=torch.int32),
             "rotary": torch.cat([angles.cos(), angles.sin()], 1).float(), "eps": 1e-6,
             "q_weight": None, "k_weight": None}
        if case["norm"]:
            s["q_weight"] = (1 + 0.2 * _randn(gen, d)).to(dtype)
            s["k_weight"] = (1 + 0.2 * _randn(gen, d)).to(dtype)
        return s
    nq, keys, first, prefix = _lengths(case)
    own_pages, shared = [-(-n // page) for n in keys], [-(-n // page) for n in prefix]
    pages = sum(own_pages) + sum(shared) + 3
    order = torch.randperm(pages, generator=gen, device=DEVICE)
    own_table, at = _page_table(own_pages, order, 0)
    s = {"op": "attend", "q": 1.5 * _randn(gen, sum(nq), hq, d), "scale": d ** -0.5, "most": max(nq),
         "k_pages": _randn(gen, pages, hkv, page, d).to(dtype).transpose(1, 2),
         "v_pages": _randn(gen, pages, hkv, page, d).to(dtype).transpose(1, 2),
         "q_first": _ints([sum(nq[:i]) for i in range(len(nq) + 1)]), "own_pages": own_table, "own_len": _ints(keys),
         "group_first": None, "prefix_pages": None, "prefix_len": None}
    s["q"] = s["q"].to(dtype)
    if prefix:
        s["prefix_pages"], at = _page_table(shared, order, at)
        s["group_first"], s["prefix_len"] = _ints(first), _ints(prefix)
    return s


# --------------------------------------------------------------------------- #
# The plain forms
# --------------------------------------------------------------------------- #
def _rotated(x, weight, s):
    """Heads [t, h, d] normed where there is a weight, then rotated, in 32 bits."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * weight.float()
    row = s["rotary"][s["positions"].long()]
    half = row.shape[1] // 2
    c, n = row[:, None, :half], row[:, None, half:]
    r, rest = x[..., :2 * half], x[..., 2 * half:]
    if s["interleaved"]:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    else:
        a, b = r[..., :half], r[..., half:]
        r = torch.cat([a * c - b * n, b * c + a * n], -1)
    return torch.cat([r, rest], -1)


def _plain_append(s):
    q = _rotated(s["q"], s["q_weight"], s).to(s["q"].dtype)
    k = _rotated(s["k"], s["k_weight"], s).to(s["k_pages"].dtype)
    page = s["k_pages"].shape[1]
    kept = s["slots"] >= 0
    at = s["slots"][kept]
    s["k_pages"][at // page, at % page] = k[kept]
    s["v_pages"][at // page, at % page] = s["v"][kept]
    return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}


def _plain_attend(s):
    """Every sequence's keys side by side, prefix first, filled up to the longest; one softmax over all."""
    q, kp, vp = s["q"], s["k_pages"], s["v_pages"]
    page, hkv, hq, d = kp.shape[1], kp.shape[2], q.shape[1], q.shape[2]
    b = s["own_len"].numel()
    first, own_len = s["q_first"].long(), s["own_len"].long()
    seq = torch.arange(b, device=q.device)
    i = torch.arange(s["own_pages"].shape[1] * page, device=q.device)
    index = s["own_pages"].long()[:, i // page].clamp(min=0) * page + i % page
    own_key, held = i.expand(b, -1), i[None] < own_len[:, None]
    if s["prefix_len"] is not None:
        group = torch.searchsorted(s["group_first"].long(), seq, right=True) - 1
        j = torch.arange(s["prefix_pages"].shape[1] * page, device=q.device)
        shared = s["prefix_pages"].long()[:, j // page].clamp(min=0) * page + j % page
        index = torch.cat([shared[group], index], 1)
        held = torch.cat([(j[None] < s["prefix_len"].long()[:, None])[group], held], 1)
        own_key = torch.cat([torch.full((b, j.numel()), -1 << 30, device=q.device), own_key], 1)
    k = kp[index // page, index % page].float().permute(0, 2, 3, 1)        # [b, hkv, d, keys]
    v = torch.where(held[..., None, None], vp[index // page, index % page].float(), 0.0).permute(0, 2, 1, 3)
    n = first[1:] - first[:-1]
    most, rep = s["most"], hq // hkv
    t = torch.arange(most, device=q.device)
    row = (first[:-1, None] + t[None]).clamp(max=q.shape[0] - 1)            # [b, most]
    x = q[row].float().view(b, most, hkv, rep, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, most * rep, d)
    score = torch.matmul(x, k.contiguous()) * s["scale"]
    seen = held[:, None] & (own_key[:, None] < (own_len - n + 1)[:, None, None] + t[None, :, None])
    seen = seen[:, None, :, None].expand(b, 1, most, rep, -1).reshape(b, 1, most * rep, -1)
    score = score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v.contiguous()) / total.clamp(min=1e-30)
    lse = (top + total.log()).view(b, hkv, most, rep).permute(0, 2, 1, 3).reshape(b, most, hq)
    out = out.view(b, hkv, most, rep, d).permute(0, 2, 1, 3, 4).reshape(b, most, hq, d)
    real = t[None] < n[:, None]
    return {"out": out[real].to(q.dtype), "lse": lse[real]}


def run(state):
    s = state
    if not own:
        return _plain_append(s) if s["op"] == "append" else _plain_attend(s)
    import paper_2607_23115_amd as g
    if s["op"] == "append":
        q = g.kv_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["slots"], q=s["q"], positions=s["positions"],
                        rotary=s["rotary"], interleaved=s["interleaved"], q_weight=s["q_weight"],
                        k_weight=s["k_weight"], eps=s["eps"])
        return {"q": q, "k_pages": s["k_pages"], "v_pages": s["v_pages"]}
    out, lse = g.prefix_attention(s["q"], s["k_pages"], s["v_pages"], s["q_first"], s["own_pages"], s["own_len"],
                                  group_first=s["group_first"], prefix_pages=s["prefix_pages"],
                                  prefix_len=s["prefix_len"], scale=s["scale"], want_lse=True)
    return {"out": out, "lse": lse}


def work(case):
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] == "append":
        t = case["t"]
        values = t * (hq + 2 * hkv) * d
        return {"bytes": 2 * 2 * values + t * (4 * case["rot"] + 12), "flops": 6 * t * (hq + hkv) * d}
    nq, keys, first, prefix = _lengths(case)
    shared = [0] * len(nq)
    for g, p in enumerate(prefix):
        shared[first[g]:first[g + 1]] = [p] * (first[g + 1] - first[g])
    pairs = sum(p + max(0, k - n + i + 1) for n, k, p in zip(nq, keys, shared) for i in range(n))
    held = sum(keys) + sum(prefix)
    return {"bytes": 2 * 2 * held * hkv * d + sum(nq) * hq * (2 * 2 * d + 4) + 4 * held // case["page"],
            "flops": 4 * pairs * hq * d}


# --------------------------------------------------------------------------- #
# In 64 bits, from the definition
# --------------------------------------------------------------------------- #
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "append":
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE),
                           _angles(case, torch.float64)[s["positions"].long()])[:, None]
        r = case["rot"]

        def heads(x, weight):
            x = x.double()
            if weight is not None:
                x = x / (x.pow(2).sum(-1, keepdim=True) / case["d"] + s["eps"]).sqrt() * weight.double()
            x = x.clone()
            pair = (slice(0, r, 2), slice(1, r, 2)) if case["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
            z = torch.complex(x[..., pair[0]], x[..., pair[1]]) * turn
            x[..., pair[0]], x[..., pair[1]] = z.real, z.imag
            return x

        q, k = heads(s["q"], s["q_weight"]), heads(s["k"], s["k_weight"])
        kp, vp = s["k_pages"].double(), s["v_pages"].double()
        token = torch.nonzero(s["slots"] >= 0).flatten()
        place = (s["slots"][token] // case["page"], s["slots"][token] % case["page"])
        kp.index_put_(place, k[token])
        vp.index_put_(place, s["v"][token].double())
        return {"q": q, "k_pages": kp, "v_pages": vp}
    nq, keys, first, prefix = _lengths(case)
    d, page, rep = case["d"], case["page"], case["hq"] // case["hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEVICE)
    group = [g for g in range(len(prefix)) for _ in range(first[g], first[g + 1])] or [None] * len(nq)
    at = 0
    for b, (n, own_keys) in enumerate(zip(nq, keys)):
        p = prefix[group[b]] if prefix else 0
        rows = [s["own_pages"][b, :-(-own_keys // page)].long()]
        counts = [own_keys]
        if p:
            rows, counts = [s["prefix_pages"][group[b], :-(-p // page)].long()] + rows, [p] + counts
        limit = p + own_keys - n + 1 + torch.arange(n, device=DEVICE)
        limit = torch.where(limit > p, limit, p)
        unseen = torch.arange(p + own_keys, device=DEVICE)[None] >= limit[:, None]
        for h in range(case["hkv"]):
            k, v = (torch.cat([x[r, :, h].reshape(-1, d)[:c].double() for r, c in zip(rows, counts)])
                    for x in (s["k_pages"], s["v_pages"]))
            for j in range(h * rep, (h + 1) * rep):
                score = (s["q"][at:at + n, j].double() @ k.T) * s["scale"]
                score[unseen] = -math.inf
                lse[at:at + n, j] = torch.logsumexp(score, 1)
                out[at:at + n, j] = torch.exp(score - lse[at:at + n, j, None].clamp(min=-1e300)) @ v
        at += n
    return {"out": out, "lse": lse}
