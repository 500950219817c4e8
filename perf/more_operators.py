"""Checking trees of drafted tokens over the paged key/value cache, and keeping the cache within a
budget: the operators in their plain form and as the library's calls.

A case is a dict of plain values; its "op" names the operator of one pass:

  tree     which drafts of its sequence each drafted token sees (itself and its ancestors), and how
           deep it is, from the drafts' parents: draft_tree()
  attend   attention of the drafts over a paged cache, a prefix of a group shared: tree_attention()
  accept   keys and values of the path that was accepted move together: kv_accept()
  weigh    the attention weight that new tokens gave each key of the cache, added up: kv_weigh()
  evict    the keys that gathered the least make room, those that stay move up: kv_evict()

A case fixes how many of everything there are: lengths are drawn from its "ragged" number, so
that the work of a pass does not depend on the seed. The seed draws the contents: keys, values,
queries, the drafts' parents, weights, which pages of the cache hold what, and in which order. Head
counts, widths and fp16 are the 7B decoder's of workloads/ (32 heads of 128), or of decoders whose
heads share keys.
"""

import math
import random

import torch

own = False
DEVICE = "cuda"
TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}


def _case(name, op, b, nq, ragged, lo=0, hi=0, hq=0, hkv=0, d=0, page=16, dtype="bf16", groups=0, prefix=0,
          path=0, keep=0, sinks=0, recent=0, fresh=False, whole=False):
    """b sequences of up to nq new tokens (of exactly nq where "whole") and lo to hi keys of their own,
    the new tokens' among them; groups that share up to "prefix" keys; path: most accepted drafts; fresh:
    the keys lie in their tokens' order, as a prompt leaves them."""
    return {"name": name, "op": op, "b": b, "nq": nq, "ragged": ragged, "lo": lo, "hi": hi, "hq": hq, "hkv": hkv,
            "d": d, "page": page, "dtype": dtype, "groups": groups, "prefix": prefix, "path": path, "keep": keep,
            "sinks": sinks, "recent": recent, "fresh": fresh, "whole": whole}


def listed():
    return [
        # One user's small tree: the smallest call, bound by latency.
        _case("tree_one_13", "tree", 1, 13, 1, whole=True),
        # A full serving batch of large trees, of sizes that differ.
        _case("tree_96x160", "tree", 96, 160, 2),
        # One user's drafts in the 7B decoder behind a conversation.
        _case("drafts_one_26", "attend", 1, 26, 3, 1047, 1047, 32, 32, 128, 16, "fp16", whole=True),
        # A batch of assistants, their drafts behind two system prompts and histories of their own.
        _case("drafts_32x64_shared", "attend", 32, 64, 4, 64, 2000, 32, 8, 128, 64, "bf16", groups=2, prefix=2048),
        # A few users with very long documents: bound by reading the cache. An odd sharing of key heads.
        _case("drafts_4x48_long", "attend", 4, 48, 5, 30000, 65531, 28, 4, 128, 64, "bf16"),
        # One user's accepted path, all heads of the 7B decoder.
        _case("accept_one", "accept", 1, 26, 6, 1047, 1047, 0, 32, 128, 16, "fp16", path=6, whole=True),
        # A large batch, wide heads.
        _case("accept_128x64", "accept", 128, 64, 7, 64, 1000, 0, 8, 256, 64, "bf16", path=20),
        # One token after a short history.
        _case("weigh_one_317", "weigh", 1, 1, 8, 317, 317, 32, 32, 128, 16, "fp16"),
        # The next tokens of a serving batch: bound by reading the keys.
        _case("weigh_64x4000", "weigh", 64, 1, 9, 500, 4000, 32, 8, 128, 64, "bf16"),
        # A whole prompt: bound by the matrix units and the exponentials.
        _case("weigh_prompt_4097", "weigh", 1, 4097, 10, 4097, 4097, 32, 8, 128, 64, "bf16", whole=True),
        # A serving batch at its budget, a few tokens over it, some sequences still below.
        _case("evict_64_at_2048", "evict", 64, 1, 11, 1990, 2112, 0, 8, 128, 64, "bf16", keep=2048, sinks=4,
              recent=256),
        # Prompts of different lengths cut down after they were read.
        _case("evict_prompts_8", "evict", 8, 1, 12, 5000, 30000, 0, 8, 128, 64, "bf16", keep=1024, sinks=4,
              recent=128, fresh=True),
    ]


def _log(rng, lo, hi):
    return lo if hi <= lo else min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["tree", "attend", "attend", "accept", "weigh", "weigh", "evict"])
    d, page = rng.choice([64, 128, 128, 256]), rng.choice([16, 32, 64, 128])
    hkv = rng.choice([1, 2, 4, 5, 8, 8, 16])
    hq = hkv * rng.choice([r for r in (1, 2, 3, 4, 4, 7, 8) if r * hkv <= 64])
    c = _case("", op, 1, 1, rng.randrange(1 << 20), 1, 1, hq, hkv, d, page, rng.choice(["fp16", "bf16"]))
    if op == "tree":
        c.update(b=_log(rng, 1, 96), nq=_log(rng, 10, 160))
        c.update(whole=c["b"] < 4)
    elif op in ("attend", "accept"):
        c.update(b=_log(rng, 1, 64), nq=_log(rng, 2, 100))
        c.update(lo=c["nq"], hi=c["nq"] + _log(rng, 1, 60000 if c["b"] <= 4 else 3000), path=_log(rng, 1, 24))
        if op == "attend" and rng.random() < 0.6:
            c.update(groups=min(c["b"], rng.choice([1, 1, 3, 8])), prefix=_log(rng, 1, 4096))
    elif op == "weigh":
        kind = rng.choice(["one", "decode", "verify", "prompt"])
        if kind == "prompt":
            n = _log(rng, 16, 3000)
            c.update(nq=n, lo=n, hi=n, whole=True)
        elif kind == "one":
            n = _log(rng, 1, 65536)
            c.update(lo=n, hi=n)
        else:
            c.update(b=_log(rng, 2, 128), nq=1 if kind == "decode" else rng.randint(2, 20))
            c.update(lo=c["nq"], hi=c["nq"] + _log(rng, 1, 3000))
    else:
        keep = _log(rng, 64, 4096)
        c.update(b=_log(rng, 1, 96), keep=keep, sinks=rng.choice([0, 1, 4]), recent=rng.randint(0, keep // 2),
                 fresh=rng.random() < 0.5)
        c.update(lo=keep // 2, hi=keep + _log(rng, 1, keep if c["b"] > 8 else 8 * keep))
    # what the plain form gathers and scores stays below the largest listed cases'
    while (c["op"] != "tree" and (c["b"] * (c["hi"] + c["prefix"]) * hkv * d > 1 << 28
                                  or hq * c["b"] * c["nq"] * (c["hi"] + c["prefix"]) > 1 << 29)):
        c["b"], c["prefix"] = max(1, c["b"] // 2), c["prefix"] // 2
        if c["b"] == 1:
            if c["op"] == "evict":
                c["hi"] = max(c["lo"], c["hi"] // 2)
            elif c["whole"]:
                c["nq"] = c["lo"] = c["hi"] = max(1, c["hi"] // 2)
            else:
                c["hi"] = max(c["nq"], c["hi"] // 2)
                c["lo"] = min(c["lo"], c["hi"])
    c["groups"] = min(c["groups"], c["b"]) if c["prefix"] else 0
    del c["name"]
    return c


def _lengths(case):
    """New tokens and own keys of each sequence, the first sequence of each group, the prefixes' lengths, the
    accepted paths (indexes among a sequence's drafts; none for a sequence that accepts nothing)."""
    rng = random.Random(case["ragged"])
    b, g = case["b"], case["groups"]
    nq = [case["nq"] if case["whole"] or case["nq"] == 1 else rng.randint(1, case["nq"]) for _ in range(b)]
    keys = [max(n, _log(rng, max(1, case["lo"]), case["hi"])) for n in nq]
    first = [0] + sorted(rng.sample(range(1, b), g - 1)) + [b] if g else [0]
    prefix = [_log(rng, max(1, case["prefix"] // 2), case["prefix"]) for _ in range(g)]
    paths = []
    for n in nq:
        m = _log(rng, 1, min(n, case["path"])) if case["path"] else 0
        if b > 1 and rng.random() < 0.05:
            m = 0
        if 2 * m <= n + 1:  # behind siblings that were not accepted
            paths.append([0] + sorted(rng.sample(range(m, n), m - 1)) if m else [])
        else:
            paths.append(list(range(m)))
    return nq, keys, first, prefix, paths


def _words(case):
    return -(-case["nq"] // 64)


def _randn(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEVICE)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEVICE)


def _offsets(counts):
    return _ints([sum(counts[:i]) for i in range(len(counts) + 1)])


def _page_table(per_row, order, at):
    """One row of page numbers for each count, filled up with -1; `order`: the cache's pages, shuffled."""
    width = max([1] + per_row)
    table = torch.full((len(per_row), width), -1, dtype=torch.int32, device=DEVICE)
    held = torch.arange(width, device=DEVICE)[None] < _ints(per_row)[:, None]
    n = sum(per_row)
    table[held] = order[at:at + n].to(torch.int32)
    return table, at + n


def _parents(nq, gen):
    """A random earlier draft of the same sequence for each, -1 for the first and a few others."""
    count = _ints(nq, torch.int64)
    i = torch.arange(sum(nq), device=DEVICE) - torch.repeat_interleave(count.cumsum(0) - count, count)
    parent = (torch.rand(len(i), generator=gen, device=DEVICE, dtype=torch.float64) * i).long()
    parent[(i == 0) | (torch.rand(len(i), generator=gen, device=DEVICE) < 0.02)] = -1
    return parent.to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    op, hq, hkv, d, page = case["op"], case["hq"], case["hkv"], case["d"], case["page"]
    nq, keys, first, prefix, paths = _lengths(case)
    s = {"op": op, "q_first": _offsets(nq), "most": case["nq"], "width": case["nq"]}
    if op in ("tree", "attend", "accept"):
        s["parent"] = _parents(nq, gen)
    if op == "accept":  # the path's drafts follow each other
        at = [sum(nq[:i]) for i in range(len(nq))]
        s["parent"][_ints([a + j for a, p in zip(at, paths) for j in p], torch.int64)] = _ints(
            [v for p in paths for v in [-1] + p[:-1] if p])
        s["leaf"] = _ints([p[-1] if p else -1 for p in paths])
    if op == "tree":
        return s
    if op in ("attend", "accept"):
        s["seen"] = _plain_tree(s)["seen"]
    dtype = TYPES[case["dtype"]]
    own_pages, shared = [-(-n // page) for n in keys], [-(-n // page) for n in prefix]
    pages = sum(own_pages) + sum(shared) + 3
    order = torch.randperm(pages, generator=gen, device=DEVICE)
    s["own_pages"], at = _page_table(own_pages, order, 0)
    s["own_len"] = _ints(keys)
    s["k_pages"] = _randn(gen, pages, hkv, page, d).to(dtype).transpose(1, 2)
    if op != "weigh":
        s["v_pages"] = _randn(gen, pages, hkv, page, d).to(dtype).transpose(1, 2)
    if op in ("attend", "weigh"):
        s["q"], s["scale"] = (1.5 * _randn(gen, sum(nq), hq, d)).to(dtype), d ** -0.5
    if op == "attend":
        s["group_first"] = s["prefix_pages"] = s["prefix_len"] = None
        if prefix:
            s["prefix_pages"], at = _page_table(shared, order, at)
            s["group_first"], s["prefix_len"] = _ints(first), _ints(prefix)
    if op == "accept":
        s["len_out"] = torch.zeros_like(s["own_len"])
    if op in ("weigh", "evict"):
        held = (torch.arange(max(keys), device=DEVICE)[None] < s["own_len"][:, None])[:, None]
        weights = -torch.rand(len(keys), hkv, max(keys), generator=gen, device=DEVICE).clamp(min=1e-6).log()
        weights[torch.rand(weights.shape, generator=gen, device=DEVICE) < 0.02] = 0.0
        where = _places(s["own_pages"], page, max(keys))
        place = (where // page)[:, None].expand_as(weights), (where % page)[:, None].expand_as(weights)
        held = held.expand_as(weights)
        at = place[0][held], torch.arange(hkv, device=DEVICE)[None, :, None].expand_as(weights)[held], place[1][held]
        s["weights"] = torch.zeros(pages, hkv, page, device=DEVICE)
        s["weights"][at] = weights[held]
        s["born"] = torch.zeros(pages, hkv, page, dtype=torch.int32, device=DEVICE)
        if op == "weigh":  # what attention would give: log of the sum of exponentials of random scores
            count = _ints(nq, torch.int64)
            t = torch.arange(sum(nq), device=DEVICE) - torch.repeat_interleave(s["q_first"][:-1].long(), count)
            sees = torch.repeat_interleave(s["own_len"].long() - count, count) + t + 1
            s["lse"] = sees.float().log()[:, None] + 0.5 * (s["q"].float().square().sum(-1) * s["scale"] ** 2)
            s["positions"] = (sees - 1).to(torch.int32)
            s["weights_out"] = torch.zeros_like(s["weights"])
        else:
            born = torch.arange(max(keys), device=DEVICE).expand_as(weights)
            if not case["fresh"]:  # places have changed hands, in each head its own
                mixed = torch.rand(weights.shape, generator=gen, device=DEVICE).masked_fill(~held, 2.0)
                born = mixed.argsort(-1).argsort(-1)
            s["born"][at] = born[held].to(torch.int32)
            s["total"] = s["own_len"].clone()
            s["weights_out"], s["born_out"] = torch.zeros_like(s["weights"]), torch.zeros_like(s["born"])
            s["len_out"] = torch.zeros_like(s["own_len"])
            s.update(keep=case["keep"], sinks=case["sinks"], recent=case["recent"])
    return s


# --------------------------------------------------------------------------- #
# The plain forms
# --------------------------------------------------------------------------- #
def _places(table, page, keys):
    """Where in the cache each row's keys are: page * page_tokens + place, of page 0 where there is none."""
    i = torch.arange(keys, device=table.device)
    return table.long()[:, (i // page).clamp(max=table.shape[1] - 1)].clamp(min=0) * page + i % page


def _plain_tree(s):
    """Who reaches whom in one step, squared until the longest path is covered."""
    parent, first, most = s["parent"].long(), s["q_first"].long(), s["most"]
    n = first[1:] - first[:-1]
    i = torch.arange(most, device=parent.device)
    real = i[None] < n[:, None]
    padded = torch.full((len(n), most), -1, dtype=torch.int64, device=parent.device)
    padded[real] = parent
    reach = ((padded[:, :, None] == i) | torch.eye(most, dtype=torch.bool, device=parent.device)).float()
    for _ in range(max(1, (most - 1).bit_length())):
        reach = (torch.matmul(reach, reach) > 0).float()
    words = -(-s["width"] // 64)
    bits = torch.zeros(len(n), most, words * 64, dtype=torch.int64, device=parent.device)
    bits[..., :most] = reach.long()
    seen = (bits.view(len(n), most, words, 64) << torch.arange(64, device=parent.device)).sum(-1)
    return {"seen": seen[real], "depth": (reach.sum(-1).long() - 1)[real].to(torch.int32)}


def _unpacked(seen, most):
    """[rows, most] truth values of the bits."""
    bits = (seen[..., None] >> torch.arange(64, device=seen.device)) & 1
    return bits.flatten(-2)[..., :most].bool()


def _plain_attend(s):
    """Every sequence's keys side by side, prefix first, filled up to the longest; one softmax over all."""
    q, kp, vp, most = s["q"], s["k_pages"], s["v_pages"], s["most"]
    page, hkv, hq, d = kp.shape[1], kp.shape[2], q.shape[1], q.shape[2]
    first, own_len = s["q_first"].long(), s["own_len"].long()
    b, n = own_len.numel(), first[1:] - first[:-1]
    i = torch.arange(s["own_pages"].shape[1] * page, device=q.device)
    index = _places(s["own_pages"], page, i.numel())
    held = i[None] < own_len[:, None]
    draft = i[None] - (own_len - n)[:, None]  # which draft a key is; below 0: none
    if s["prefix_len"] is not None:
        group = torch.searchsorted(s["group_first"].long(), torch.arange(b, device=q.device), right=True) - 1
        j = torch.arange(s["prefix_pages"].shape[1] * page, device=q.device)
        index = torch.cat([_places(s["prefix_pages"], page, j.numel())[group], index], 1)
        held = torch.cat([(j[None] < s["prefix_len"].long()[:, None])[group], held], 1)
        draft = torch.cat([torch.full((b, j.numel()), -1, device=q.device), draft], 1)
    k = kp[index // page, index % page].float().permute(0, 2, 3, 1)        # [b, hkv, d, keys]
    v = vp[index // page, index % page].float().permute(0, 2, 1, 3)
    t, rep = torch.arange(most, device=q.device), hq // hkv
    row = (first[:-1, None] + t[None]).clamp(max=q.shape[0] - 1)            # [b, most]
    x = q[row].float().view(b, most, hkv, rep, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, most * rep, d)
    score = torch.matmul(x, k.contiguous()) * s["scale"]
    bits = torch.nn.functional.pad(_unpacked(s["seen"], most)[row], (1, 0), value=True)  # what is no draft is seen
    sees = bits.gather(2, (draft + 1).clamp(0, most)[:, None].expand(-1, most, -1)) & held[:, None]
    sees = sees[:, None, :, None].expand(b, 1, most, rep, -1).reshape(b, 1, most * rep, -1)
    score = score.masked_fill_(~sees, -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-1e30)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v.contiguous()) / total.clamp(min=1e-30)
    lse = (top + total.log()).view(b, hkv, most, rep).permute(0, 2, 1, 3).reshape(b, most, hq)
    out = out.view(b, hkv, most, rep, d).permute(0, 2, 1, 3, 4).reshape(b, most, hq, d)
    real = t[None] < n[:, None]
    return {"out": out[real].to(q.dtype), "lse": lse[real]}


def _plain_accept(s):
    kp, vp, first, own_len = s["k_pages"], s["v_pages"], s["q_first"].long(), s["own_len"].long()
    page, base = kp.shape[1], own_len - (first[1:] - first[:-1])
    leaf = s["leaf"].long()
    row = (first[:-1] + leaf.clamp(min=0)).clamp(max=s["seen"].shape[0] - 1)
    path = _unpacked(s["seen"][row], s["most"]) & (leaf >= 0)[:, None]
    seq, draft = path.nonzero(as_tuple=True)
    to = (path.cumsum(1) - 1)[seq, draft]
    where = _places(s["own_pages"], page, s["own_pages"].shape[1] * page)
    src, dst = where[seq, base[seq] + draft], where[seq, base[seq] + to]
    kp[dst // page, dst % page] = kp[src // page, src % page]
    vp[dst // page, dst % page] = vp[src // page, src % page]
    s["len_out"].copy_(base + path.sum(1))
    return {"k_pages": kp, "v_pages": vp, "len_out": s["len_out"]}


def _plain_weigh(s):
    q, kp, most = s["q"], s["k_pages"], s["most"]
    page, hkv, hq, d = kp.shape[1], kp.shape[2], q.shape[1], q.shape[2]
    first, own_len = s["q_first"].long(), s["own_len"].long()
    b, n, rep = own_len.numel(), first[1:] - first[:-1], hq // kp.shape[2]
    i = torch.arange(s["own_pages"].shape[1] * page, device=q.device)
    where = _places(s["own_pages"], page, i.numel())
    k = kp[where // page, where % page].float().permute(0, 2, 3, 1)        # [b, hkv, d, keys]
    t = torch.arange(most, device=q.device)
    real = t[None] < n[:, None]
    row = (first[:-1, None] + t[None]).clamp(max=q.shape[0] - 1)            # [b, most]
    x = q[row].float().view(b, most, hkv, rep, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, most * rep, d)
    lse = s["lse"][row].view(b, most, hkv, rep).permute(0, 2, 1, 3).reshape(b, hkv, most * rep, 1)
    p = (torch.matmul(x, k.contiguous()) * s["scale"]).sub_(lse).exp_()
    sees = (i[None, None] < (own_len - n + 1)[:, None, None] + t[None, :, None]) & real[..., None]
    sees = sees[:, None, :, None].expand(b, 1, most, rep, -1).reshape(b, 1, most * rep, -1)
    sums = p.masked_fill_(~sees, 0.0).sum(2)                                # [b, hkv, keys]
    held, new = i[None] < own_len[:, None], i[None] >= (own_len - n)[:, None]
    seq, key = held.nonzero(as_tuple=True)
    at = where[seq, key] // page, where[seq, key] % page
    old = torch.where(new[seq, key][:, None], 0.0, s["weights"].transpose(1, 2)[at])
    s["weights_out"].transpose(1, 2)[at] = old + sums.transpose(1, 2)[seq, key]
    seq, key = (held & new).nonzero(as_tuple=True)
    at = where[seq, key] // page, where[seq, key] % page
    token = first[seq] + key - (own_len - n)[seq]
    s["born"].transpose(1, 2)[at] = s["positions"][token][:, None].expand(-1, hkv)
    return {"weights": s["weights_out"], "born": s["born"]}


def _plain_evict(s):
    kp, vp, keep = s["k_pages"], s["v_pages"], s["keep"]
    page, hkv, own_len = kp.shape[1], kp.shape[2], s["own_len"].long()
    i = torch.arange(s["own_pages"].shape[1] * page, device=kp.device)
    where = _places(s["own_pages"], page, i.numel())
    held = (i[None] < own_len[:, None])[:, None]                            # [b, 1, keys]
    weight = s["weights"][where // page, :, where % page].transpose(1, 2)   # [b, hkv, keys]
    born = s["born"][where // page, :, where % page].transpose(1, 2)
    safe = (born < s["sinks"]) | (born >= (s["total"] - s["recent"])[:, None, None])
    weight = weight.masked_fill(safe, math.inf).masked_fill(~held, -math.inf)
    order = weight.sort(dim=-1, descending=True, stable=True)[1]            # ties: the lowest place first
    kept = torch.zeros_like(weight, dtype=torch.bool).scatter_(-1, order[..., :keep], True) & held
    room, moved = held & ~kept & (i < keep), kept & (i >= keep)             # as many of both, in order
    seq, head, to = room.nonzero(as_tuple=True)
    dst, src = where[seq, to], where[seq, moved.nonzero(as_tuple=True)[2]]
    kp[dst // page, dst % page, head] = kp[src // page, src % page, head]
    vp[dst // page, dst % page, head] = vp[src // page, src % page, head]
    seq1, to1 = (held[:, 0] & (i < keep)).nonzero(as_tuple=True)
    at = where[seq1, to1] // page, where[seq1, to1] % page
    for x, y in ((s["weights"], s["weights_out"]), (s["born"], s["born_out"])):
        y.transpose(1, 2)[at] = x.transpose(1, 2)[at]
        y[dst // page, head, dst % page] = x[src // page, head, src % page]
    s["len_out"].copy_(own_len.clamp(max=keep))
    return {"k_pages": kp, "v_pages": vp, "weights": s["weights_out"], "born": s["born_out"], "len_out": s["len_out"]}


def run(state):
    s, op = state, state["op"]
    if not own:
        return {"tree": _plain_tree, "attend": _plain_attend, "accept": _plain_accept, "weigh": _plain_weigh,
                "evict": _plain_evict}[op](s)
    import paper_2607_23115_amd as g
    if op == "tree":
        seen, depth = g.draft_tree(s["parent"], s["q_first"], s["width"])
        return {"seen": seen, "depth": depth}
    if op == "attend":
        out, lse = g.tree_attention(s["q"], s["k_pages"], s["v_pages"], s["q_first"], s["seen"], s["own_pages"],
                                    s["own_len"], group_first=s["group_first"], prefix_pages=s["prefix_pages"],
                                    prefix_len=s["prefix_len"], scale=s["scale"], want_lse=True)
        return {"out": out, "lse": lse}
    if op == "accept":
        len_out = g.kv_accept(s["k_pages"], s["v_pages"], s["q_first"], s["seen"], s["leaf"], s["own_pages"],
                              s["own_len"], len_out=s["len_out"])
        return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "len_out": len_out}
    if op == "weigh":
        weights = g.kv_weigh(s["q"], s["k_pages"], s["q_first"], s["own_pages"], s["own_len"], s["lse"], s["weights"],
                             born=s["born"], positions=s["positions"], weights_out=s["weights_out"], scale=s["scale"])
        return {"weights": weights, "born": s["born"]}
    len_out = g.kv_evict(s["k_pages"], s["v_pages"], s["own_pages"], s["own_len"], s["weights"], s["born"], s["total"],
                         s["keep"], sinks=s["sinks"], recent=s["recent"], weights_out=s["weights_out"],
                         born_out=s["born_out"], len_out=s["len_out"])
    return {"k_pages": s["k_pages"], "v_pages": s["v_pages"], "weights": s["weights_out"], "born": s["born_out"],
            "len_out": len_out}


def work(case):
    op, hq, hkv, d = case["op"], case["hq"], case["hkv"], case["d"]
    nq, keys, first, prefix, paths = _lengths(case)
    tokens, b = sum(nq), len(nq)
    if op == "tree":  # a parent read, bits and depth written
        return {"bytes": tokens * (4 + 8 * _words(case) + 4) + 4 * (b + 1), "flops": 0}
    tables = 4 * sum(keys) // case["page"] + 8 * b
    if op == "attend":
        shared = [0] * b
        for g, p in enumerate(prefix):
            shared[first[g]:first[g + 1]] = [p] * (first[g + 1] - first[g])
        # of its sequence's drafts a token sees about as many as it is deep: few
        pairs = sum(n * (p + k - n) + n * int(1 + math.log(n)) for n, k, p in zip(nq, keys, shared))
        return {"bytes": 4 * (sum(keys) + sum(prefix)) * hkv * d + tokens * (hq * (4 * d + 4) + 8 * _words(case)) +
                tables, "flops": 4 * pairs * hq * d}
    if op == "accept":  # what moves is read and written
        moved = sum(j != e for p in paths for e, j in enumerate(p))
        return {"bytes": moved * hkv * d * 2 * 2 * 2 + b * (8 * _words(case) + 16), "flops": 0}
    if op == "weigh":
        pairs = sum(n * (k - n) + n * (n + 1) // 2 for n, k in zip(nq, keys))
        return {"bytes": sum(keys) * hkv * (2 * d + 4) + sum(k - n for n, k in zip(nq, keys)) * hkv * 4 +
                tokens * (hq * (2 * d + 4) + 4 + 4 * hkv) + tables, "flops": 2 * pairs * hq * d}
    # evict: all weights and births read, those of the kept written, and the keys that move, of
    # random weights on average
    moved, kept = 0.0, 0
    for k in keys:
        keep, safe = min(k, case["keep"]), min(k, case["sinks"] + case["recent"])
        rest = (keep - safe) / (k - safe) if k > keep > safe else float(k <= keep)
        over = k - keep
        behind = min(over, case["recent"] if case["fresh"] else safe * over / k)  # of the safe ones
        moved += behind + (over - behind) * rest
        kept += keep
    return {"bytes": int(hkv * (8 * sum(keys) + 8 * kept + moved * d * 2 * 2 * 2)) + tables, "flops": 0}


# --------------------------------------------------------------------------- #
# In 64 bits, from the definition
# --------------------------------------------------------------------------- #
def exact(case, seed):
    s = prepare(case, seed)
    op, d, page, hkv = case["op"], case["d"], case["page"], case["hkv"]
    nq, keys, first, prefix, paths = _lengths(case)
    if op == "tree":
        seen, depth, at, parent = [], [], 0, s["parent"].tolist()
        for n in nq:
            for i in range(n):
                up, j, steps = 0, i, -1
                while j >= 0:
                    up |= 1 << j
                    j = parent[at + j]
                    steps += 1
                words = [(up >> (64 * w)) & ((1 << 64) - 1) for w in range(_words(case))]
                seen.append([w - (1 << 64) if w >> 63 else w for w in words])
                depth.append(steps)
            at += n
        return {"seen": _ints(seen, torch.int64), "depth": _ints(depth)}
    rows = [s["own_pages"][b, :-(-k // page)].long() for b, k in enumerate(keys)]

    def of(x, b, h):  # keys or values of a sequence and head, in order
        return x[rows[b], :, h].reshape(-1, d)[:keys[b]]

    if op == "attend":
        rep = case["hq"] // hkv
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
        lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device=DEVICE)
        group = [g for g in range(len(prefix)) for _ in range(first[g], first[g + 1])]
        seen, at = s["seen"].tolist(), 0
        for b, n in enumerate(nq):
            p = prefix[group[b]] if prefix else 0
            bits = [sum((w & ((1 << 64) - 1)) << (64 * k) for k, w in enumerate(r)) for r in seen[at:at + n]]
            unseen = torch.zeros(n, p + keys[b], dtype=torch.bool, device=DEVICE)
            unseen[:, p + keys[b] - n:] = _ints([[not (r >> j) & 1 for j in range(n)] for r in bits], torch.bool)
            for h in range(hkv):
                k, v = of(s["k_pages"], b, h).double(), of(s["v_pages"], b, h).double()
                if p:
                    r = s["prefix_pages"][group[b], :-(-p // page)].long()
                    k, v = (torch.cat([x[r, :, h].reshape(-1, d)[:p].double(), y])
                            for x, y in ((s["k_pages"], k), (s["v_pages"], v)))
                for j in range(h * rep, (h + 1) * rep):
                    score = (s["q"][at:at + n, j].double() @ k.T) * s["scale"]
                    score[unseen] = -math.inf
                    lse[at:at + n, j] = torch.logsumexp(score, 1)
                    out[at:at + n, j] = torch.softmax(score, 1) @ v
            at += n
        return {"out": out, "lse": lse}
    if op == "weigh":
        rep, at = case["hq"] // hkv, 0
        weights, born = torch.zeros_like(s["weights"], dtype=torch.float64), s["born"]
        for b, n in enumerate(nq):
            base = keys[b] - n
            j = torch.arange(keys[b], device=DEVICE)
            where = rows[b][j // page], j % page
            late = j[None] > base + torch.arange(n, device=DEVICE)[:, None]
            for h in range(hkv):
                k = of(s["k_pages"], b, h).double().T.contiguous()
                total = torch.zeros(keys[b], dtype=torch.float64, device=DEVICE)
                total[:base] = s["weights"][where[0], h, where[1]][:base].double()
                for i in range(h * rep, (h + 1) * rep):
                    score = (s["q"][at:at + n, i].double() @ k) * s["scale"]
                    total += torch.exp(score - s["lse"][at:at + n, i, None].double()).masked_fill_(late, 0.0).sum(0)
                weights[where[0], h, where[1]] = total
                born[where[0][base:], h, where[1][base:]] = s["positions"][at:at + n]
            at += n
        return {"weights": weights, "born": born}
    kp, vp, length = s["k_pages"].clone(), s["v_pages"].clone(), list(keys)
    if op == "accept":
        for b, path in enumerate(paths):
            base = keys[b] - nq[b]
            src = _ints([base + j for j in path], torch.int64)
            dst = base + torch.arange(len(path), device=DEVICE)
            for x, y in ((s["k_pages"], kp), (s["v_pages"], vp)):
                y[rows[b][dst // page], dst % page] = x[rows[b][src // page], src % page]
            length[b] = base + len(path)
        return {"k_pages": kp.double(), "v_pages": vp.double(), "len_out": _ints(length)}
    weights, born = torch.zeros_like(s["weights"], dtype=torch.float64), torch.zeros_like(s["born"])
    for b, n in enumerate(keys):
        keep = min(n, case["keep"])
        for h in range(hkv):
            w, t = (s[x][rows[b], h].reshape(-1)[:n] for x in ("weights", "born"))
            safe = (t < case["sinks"]) | (t >= n - case["recent"])
            rank = sorted(zip((~safe).tolist(), (-w).tolist(), range(n)))
            rank = [(0, 0.0, i) if not r else (1, v, i) for r, v, i in rank]
            kept = {i for _, _, i in sorted(rank)[:keep]}
            room, behind = [i for i in range(keep) if i not in kept], sorted(i for i in kept if i >= keep)
            src = torch.arange(keep, device=DEVICE)
            src[_ints(room, torch.int64)] = _ints(behind, torch.int64)
            dst = torch.arange(keep, device=DEVICE)
            dst, src = (rows[b][dst // page], dst % page), (rows[b][src // page], src % page)
            for x, y in ((s["k_pages"], kp), (s["v_pages"], vp)):
                y[dst[0], dst[1], h] = x[src[0], src[1], h]
            weights[dst[0], h, dst[1]] = s["weights"][src[0], h, src[1]].double()
            born[dst[0], h, dst[1]] = s["born"][src[0], h, src[1]]
        length[b] = keep
    return {"k_pages": kp.double(), "v_pages": vp.double(), "weights": weights, "born": born, "len_out": _ints(length)}
