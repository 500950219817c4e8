"""prefix_attention on the GPU against 64-bit arithmetic on the CPU."""

import math

import pytest
import torch

import kv_reference as R
import paper_2607_23115_amd as g
from gpu_util import say

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    torch.cuda.init()


def i32(x):
    return torch.tensor(x, dtype=torch.int32)


class Case:
    """A ragged batch on the CPU. n: new tokens of each sequence, own: its keys; groups: (first
    sequence, end, prefix keys), in order. Whatever nobody may see is NaN."""

    def __init__(self, n, own, groups, hq, hkv, d, page, dtype, seed=0, head_major=True, pad_tokens=0, spread=1.0):
        gen = torch.Generator().manual_seed(seed)
        count = lambda keys: -(-keys // page)  # noqa: E731
        pages = sum(map(count, own)) + sum(count(p) for _, _, p in groups) + 2
        order = torch.randperm(pages, generator=gen).tolist()
        self.kp, self.vp = (torch.full((pages, page, hkv, d), math.nan) for _ in range(2))

        def table(counts):
            rows = torch.full((len(counts), max([1] + [count(c) for c in counts]) + 1), -1, dtype=torch.int32)
            for r, keys in enumerate(counts):
                for j in range(count(keys)):
                    rows[r, j] = order.pop()
                    m = min(page, keys - j * page)
                    self.kp[rows[r, j], :m] = torch.randn(m, hkv, d, generator=gen) * spread
                    self.vp[rows[r, j], :m] = torch.randn(m, hkv, d, generator=gen)
            return rows

        self.own_pages, self.own_len = table(own), i32(own)
        self.q_first = i32([sum(n[:i]) for i in range(len(n) + 1)])
        self.group_first = self.prefix_pages = self.prefix_len = None
        if groups:
            # sequences outside any group lie before the first and after the last, or in a group
            # of no prefix
            assert all(a[1] == b[0] for a, b in zip(groups, groups[1:]))
            self.group_first = i32([groups[0][0]] + [b for _, b, _ in groups])
            self.prefix_pages, self.prefix_len = table([p for _, _, p in groups]), i32([p for _, _, p in groups])
        self.kp, self.vp = self.kp.to(dtype), self.vp.to(dtype)
        self.q = torch.randn(sum(n) + pad_tokens, hq, d, generator=gen).to(dtype)
        self.head_major, self.scale = head_major, None
        self.what = (f"n={n if len(n) < 9 else len(n)} own={own if len(own) < 9 else len(own)} groups={groups} "
                     f"heads={hq}/{hkv} d={d} page={page} {dtype}")

    def arguments(self):
        def pages(t):
            return (t.transpose(1, 2).contiguous().cuda().transpose(1, 2) if self.head_major else t.cuda())
        dev = lambda t: None if t is None else t.cuda()  # noqa: E731
        return {"q": self.q.cuda(), "k_pages": pages(self.kp), "v_pages": pages(self.vp),
                "q_first": dev(self.q_first), "own_pages": dev(self.own_pages), "own_len": dev(self.own_len),
                "group_first": dev(self.group_first), "prefix_pages": dev(self.prefix_pages),
                "prefix_len": dev(self.prefix_len), "scale": self.scale}

    def want(self):
        return R.attention(self.q, self.kp, self.vp, self.q_first, self.own_pages, self.own_len, self.group_first,
                           self.prefix_pages, self.prefix_len, self.scale)

    def check(self, **more):
        say("prefix_attention", self.what)
        out, lse = g.prefix_attention(**{**self.arguments(), **more}, want_lse=True)
        torch.cuda.synchronize()
        o, l, o_tol, l_tol = self.want()
        R.near(lse, l, l_tol, "lse")
        R.near(out, o, o_tol, "out")
        return out, lse


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_types_and_widths(dtype, d):
    Case([1, 1, 1, 1], [1, 17, 70, 200], [(0, 3, 100)], 8, 2, d, 16, dtype).check()
    Case([5, 40, 1], [5, 60, 300], [], 4, 2, d, 32, dtype).check()
    Case([33, 70], [50, 70], [(0, 2, 75)], 4, 1, d, 16, dtype).check()


@pytest.mark.parametrize("hq,hkv", [(1, 1), (5, 5), (3, 1), (7, 1), (28, 4), (32, 32), (24, 8), (40, 2), (17, 1)])
def test_heads(hq, hkv):
    Case([1, 3, 1], [40, 33, 1], [(0, 2, 50)], hq, hkv, 64, 16, BF16, seed=hq).check()


@pytest.mark.parametrize("page", [16, 64, 256, 4096])
@pytest.mark.parametrize("head_major", [False, True])
def test_pages(page, head_major):
    Case([1, 2], [page + 1, 2 * page - 1], [(0, 2, page)], 4, 2, 128, page, F16, head_major=head_major).check()


@pytest.mark.parametrize("own", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 1000, 5001])
def test_one_token_of_one_sequence(own):
    Case([1], [own], [], 4, 1, 128, 16, BF16, seed=own).check()


@pytest.mark.parametrize("prefix", [0, 1, 63, 64, 65, 500, 3000])
def test_prefix_lengths(prefix):
    Case([1] * 5, [0, 1, 9, 64, 130], [(0, 5, prefix)], 8, 2, 64, 16, F16, seed=prefix).check()


def test_rows_that_see_nothing():
    """Sequences with fewer keys than new tokens, with none, and without tokens; tokens that no
    sequence has."""
    c = Case([4, 3, 0, 6, 2], [2, 0, 5, 6, 1], [], 4, 2, 64, 16, F16, pad_tokens=5)
    out, lse = c.check()
    assert (out[-5:] == 0).all() and (lse[-5:] == -math.inf).all()
    assert (out[:2] == 0).all() and (lse[4:7] == -math.inf).all()
    Case([4, 3, 0, 6], [2, 0, 5, 6], [(0, 4, 20)], 4, 2, 64, 16, F16, pad_tokens=2).check()
    Case([0, 0], [3, 0], [(0, 2, 8)], 2, 2, 64, 16, BF16, pad_tokens=1).check()


def test_groups():
    """A group without a prefix, one of one sequence, one whose sequences have no tokens, and
    sequences before and after all groups."""
    n = [1, 2, 1, 1, 1, 0, 0, 3, 1, 1]
    own = [3, 40, 7, 0, 90, 4, 0, 20, 66, 5]
    Case(n, own, [(1, 3, 0), (3, 4, 130), (4, 5, 77), (5, 7, 33), (7, 9, 200)], 6, 2, 128, 16, BF16).check()
    Case(n, own, [(0, 10, 150)], 6, 2, 128, 32, F16).check()
    Case(n, own, [(2, 2, 50), (2, 8, 50), (8, 8, 10)], 6, 2, 64, 16, F16).check()


@pytest.mark.parametrize("n,own,prefix", [(16, 16, 0), (64, 64, 0), (65, 65, 0), (127, 130, 0), (200, 333, 0),
                                          (300, 300, 100), (130, 129, 40), (257, 500, 64)])
def test_prompts(n, own, prefix):
    """Many tokens of a sequence, alone and as two sequences behind one prefix."""
    Case([n], [own], [(0, 1, prefix)] if prefix else [], 4, 2, 64, 16, BF16, seed=n).check()
    Case([n, n // 2], [own, n // 2], [(0, 2, prefix)], 2, 1, 128, 32, F16, seed=n).check()


def test_prompts_of_256_wide_heads():
    Case([150, 7, 1], [150, 300, 30], [(0, 3, 90)], 3, 1, 256, 16, BF16).check()
    Case([90], [200], [], 2, 2, 256, 64, F16).check()


def test_a_mixed_batch():
    """Prompts and single tokens in one batch, in groups and out of them."""
    Case([1, 200, 1, 33, 1, 1, 90], [600, 200, 1, 50, 129, 64, 400], [(0, 3, 70), (3, 7, 300)], 8, 2, 128, 32,
         BF16).check()


def test_more_sequences_than_a_plan_round():
    """Above 1,024 sequences and items the plan goes round its loops more than once."""
    gen = torch.Generator().manual_seed(3)
    own = torch.randint(0, 40, (1500,), generator=gen).tolist()
    n = torch.randint(0, 3, (1500,), generator=gen).tolist()
    Case(n, own, [(i, i + 3, 5 + i % 30) for i in range(0, 1200, 3)], 2, 1, 64, 16, F16).check()


def test_many_pieces():
    """One row over more chunks than the join reads at once, and behind a long prefix."""
    Case([1], [20000], [], 1, 1, 64, 64, BF16).check()
    Case([1, 1, 1], [3000, 10, 700], [(0, 3, 9000)], 2, 1, 64, 128, F16).check()


@pytest.mark.parametrize("spread", [0.0, 20.0])
def test_flat_and_peaked_scores(spread):
    Case([1, 30], [300, 100], [(0, 2, 200)], 4, 2, 128, 16, F16, spread=spread).check()


def test_scale_and_strided_queries():
    c = Case([1, 4, 1], [40, 50, 3], [(0, 2, 30)], 4, 2, 64, 16, BF16)
    c.scale = 0.7
    wide = torch.randn(c.q.shape[0], 10, 64).to(BF16)
    wide[:, 3:7] = c.q
    c.check(q=wide.cuda()[:, 3:7])
    c.scale = -0.2
    c.check()


def test_a_scale_of_zero_takes_the_mean_of_what_is_seen():
    for n, own, prefix in ((1, 70, 40), (100, 130, 75), (150, 100, 0)):
        c = Case([n, 1], [own, 3], [(0, 2, prefix)], 4, 2, 64, 16, BF16)
        c.scale = 0.0
        c.check()


def test_later_keys_and_values_may_be_anything():
    """Keys and values of a sequence's later tokens hold NaN and infinities: earlier tokens of
    the same call do not see them, later ones do."""
    for n, own, first in ((6, 20, 17), (80, 100, 60), (200, 200, 120)):
        c = Case([n], [own], [], 4, 2, 64, 16, BF16)
        flat = lambda x: x[c.own_pages[0, :-(-own // 16)].long()].reshape(-1, 2, 64)  # noqa: E731
        kk, vv = flat(c.kp), flat(c.vp)
        vv[first, 0, 3], vv[first, 1, 60], vv[first + 1, 0, 3] = math.inf, math.nan, -math.inf
        vv[own - 1, 1, 7] = -math.inf
        kk[own - 2, 0] = math.nan
        for x, y in ((c.kp, kk), (c.vp, vv)):
            x[c.own_pages[0, :-(-own // 16)].long()] = y.view(-1, 16, 2, 64)
        o, l, o_tol, l_tol = c.want()
        say("prefix_attention", "special values", c.what)
        out, lse = g.prefix_attention(**c.arguments(), want_lse=True)
        out, lse = out.cpu().double(), lse.cpu().double()
        at = first - (own - n)  # the first token that sees them
        fine = torch.isfinite(o[:at])
        assert fine.all() and bool(((out - o).abs()[:at] <= o_tol[:at]).all())
        assert bool(((lse - l).abs()[:at] <= l_tol[:at]).all())
        # the others: what the definition makes infinite is so, untouched dimensions hold
        assert torch.equal(torch.isnan(out), torch.isnan(o)) and torch.equal(torch.isposinf(out), torch.isposinf(o))
        assert torch.equal(torch.isneginf(out), torch.isneginf(o)) and torch.equal(torch.isnan(lse), torch.isnan(l))
        seen = torch.isfinite(o)
        assert bool(((out - o).abs()[seen] <= o_tol[seen]).all())


def test_pages_that_the_cache_does_not_have_are_not_seen():
    c = Case([1, 2, 100], [100, 60, 130], [(0, 2, 90)], 4, 2, 64, 16, F16)
    c.own_pages[0, 2], c.own_pages[1, 0], c.prefix_pages[0, 3] = -1, c.kp.shape[0], 1 << 30
    c.own_pages[2, 5] = -7
    c.check()


def test_lengths_and_offsets_out_of_range():
    """Lengths beyond the tables and below zero, offsets that fall or pass the end: taken as the
    nearest that makes sense, and nothing outside the tensors is touched."""
    c = Case([1, 1, 2], [20, 20, 20], [(0, 3, 30)], 2, 1, 64, 16, F16)
    full = c.own_pages[:, :2].clone()
    a = {**c.arguments(), "own_pages": full.cuda().contiguous()}
    say("prefix_attention", "lengths out of range")
    c.kp[torch.isnan(c.kp)] = 0.5
    c.vp[torch.isnan(c.vp)] = 0.25
    a.update({k: x for k, x in c.arguments().items() if k in ("k_pages", "v_pages")})
    long = g.prefix_attention(**{**a, "own_len": i32([1 << 30, -5, 20]).cuda()})[0]
    want = g.prefix_attention(**{**a, "own_len": i32([32, 0, 20]).cuda()})[0]
    assert torch.equal(long, want)
    odd = g.prefix_attention(**{**a, "q_first": i32([-3, 1, 0, 99]).cuda()})[0]
    want = g.prefix_attention(**{**a, "q_first": i32([0, 1, 1, 4]).cuda()})[0]
    assert torch.equal(odd, want)
    odd = g.prefix_attention(**{**a, "group_first": i32([-1, 50]).cuda()})[0]
    want = g.prefix_attention(**{**a, "group_first": i32([0, 3]).cuda()})[0]
    assert torch.equal(odd, want)


def test_a_cache_beyond_32_bit_offsets():
    pages, page, d = (1 << 32) // (4096 * 128) + 3, 4096, 128
    say("prefix_attention large cache", pages)
    kp = torch.empty(pages, page, 1, d, dtype=BF16, device="cuda")
    vp = torch.empty_like(kp)
    k, v = (torch.randn(100, 1, d).to(BF16) for _ in range(2))
    for i in (0, pages - 1):
        kp[i].fill_(math.nan)
        vp[i].fill_(math.nan)
    kp[-1, :100], vp[-1, :100] = k.cuda(), v.cuda()
    q = torch.randn(1, 4, d).to(BF16)
    one = i32([0, 1])
    out, _ = g.prefix_attention(q.cuda(), kp, vp, one.cuda(), i32([[pages - 1]]).cuda(), i32([100]).cuda())
    small = torch.full((1, page, 1, d), math.nan, dtype=BF16)
    sv = small.clone()
    small[0, :100], sv[0, :100] = k, v
    o, _, o_tol, _ = R.attention(q, small, sv, one, i32([[0]]), i32([100]))
    R.near(out, o, o_tol, "out")


def test_the_same_call_twice_gives_the_same_bits():
    c = Case([1, 30, 1, 5], [900, 300, 44, 2000], [(0, 4, 700)], 8, 2, 128, 16, BF16)
    a = c.arguments()
    x, xl = g.prefix_attention(**a, want_lse=True)
    for _ in range(3):
        y, yl = g.prefix_attention(**a, want_lse=True)
        assert torch.equal(x, y) and torch.equal(xl, yl)


def test_a_captured_call_follows_lengths_and_pages():
    c = Case([1, 1, 3], [200, 90, 40], [(0, 2, 300)], 8, 2, 128, 16, BF16)
    a = c.arguments()
    a["k_pages"][torch.isnan(a["k_pages"])] = 0.5
    a["v_pages"][torch.isnan(a["v_pages"])] = 0.25
    out, lse = torch.empty_like(a["q"]), torch.empty(a["q"].shape[:2], device="cuda")
    ws = g.prefix_attention_workspace(a["k_pages"], a["v_pages"], 5, 8, 3, 1)
    say("prefix_attention graph")
    g.prefix_attention(**a, out=out, lse=lse, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.prefix_attention(**a, out=out, lse=lse, ws=ws)
    for own, prefix in (([200, 90, 40], 300), ([3, 90, 0], 0), ([208, 1, 48], 17), ([0, 0, 0], 290)):
        a["own_len"].copy_(i32(own))
        a["prefix_len"].copy_(i32([prefix]))
        a["own_pages"].copy_(a["own_pages"].flip(0).clamp(min=0))
        want, want_l = g.prefix_attention(**a, want_lse=True)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_l)
        ws.fill_(255)  # scratch: a later call does not depend on what is there


def test_on_another_stream():
    c = Case([1, 30, 1], [900, 300, 44], [(0, 3, 700)], 8, 2, 64, 16, F16)
    a = c.arguments()
    want, _ = g.prefix_attention(**a)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    say("prefix_attention stream")
    got, lse = g.prefix_attention(**a, stream=side)
    side.synchronize()
    assert lse is None and torch.equal(got, want)


def refused(message, **kw):
    c = Case([1, 1], [5, 6], [(0, 2, 7)], 4, 2, 64, 16, F16)
    a = c.arguments()
    out = torch.full_like(a["q"], 3.0)
    a["out"] = out
    a.update({n: x(a) if callable(x) else x for n, x in kw.items()})
    with pytest.raises((ValueError, g.GleamError), match=message):
        g.prefix_attention(**a)
    torch.cuda.synchronize()
    assert (out == 3).all()


def test_refusals():
    refused("q must be", q=lambda a: a["q"].float())
    refused("q must be", q=lambda a: a["q"][0])
    refused("on the GPU", q=lambda a: a["q"].cpu())
    refused("multiple of kv_heads", q=lambda a: a["q"][:, :3].contiguous(), out=None)
    refused("q_first holds 2", q_first=lambda a: a["q_first"][:2])
    refused("own_len must be", own_len=lambda a: a["own_len"].long())
    refused("own_pages must be", own_pages=lambda a: a["own_pages"][:1])
    refused("prefix_len is required", prefix_len=None)
    refused("group_first is required", group_first=None)
    refused("prefix_pages is required", prefix_pages=None)
    refused("prefix_pages must be", prefix_pages=lambda a: a["prefix_pages"][:0])
    refused("head_dim must be 64, 128 or 256", q=lambda a: a["q"][..., :32], out=None,
            k_pages=lambda a: a["k_pages"][..., :32], v_pages=lambda a: a["v_pages"][..., :32])
    refused("page_tokens", k_pages=lambda a: a["k_pages"][:, :8], v_pages=lambda a: a["v_pages"][:, :8])
    refused("workspace of 256 bytes", ws=lambda a: torch.empty(256, dtype=torch.uint8, device="cuda"))
    refused("256-byte aligned", ws=lambda a: torch.empty(1 << 28, dtype=torch.uint8, device="cuda")[16:])
    refused("out and q differ", out=lambda a: a["q"][:1].clone())
    refused("lse must be", lse=lambda a: torch.empty(2, 3, device="cuda"))
    refused("contiguous", out=lambda a: a["q"].transpose(0, 1).contiguous().transpose(0, 1))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n", [1, 5, 16, 32, 40])
def test_infinities_beside_a_page_that_is_missing(n, dtype):
    """Of 32 keys that are looked up together one page of 16 is missing; what the other one holds
    reaches the rows that see it, infinities and NaN included."""
    c = Case([n], [140], [], 4, 2, 64, 16, dtype, seed=n)
    pages = c.own_pages[0].clone()
    c.vp[pages[3], 2, 0, 3] = math.inf     # key 50, behind a missing page
    c.vp[pages[3], 12, 1, 9] = math.nan
    c.vp[pages[4], 0, 1, 20] = -math.inf   # key 64, before one
    c.vp[pages[8], 11, 0, 33] = math.inf   # the last key
    c.own_pages[0, 2], c.own_pages[0, 5] = -1, c.kp.shape[0]
    c.check()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n", [1, 100])
def test_a_scale_of_zero_keeps_queries_that_are_not_finite(n, dtype):
    c = Case([n, 2], [130, 3], [(0, 2, 40)], 4, 2, 64, 16, dtype)
    c.q[0, 1, 5], c.q[n // 2, 2, 63] = math.nan, math.inf
    c.scale = 0.0
    c.check()


@pytest.mark.parametrize("n", [1, 40, 70])
def test_many_small_weights_of_fp16(n):
    """Each wave meets keys that outweigh every other one by 2^25.2, and tens of thousands of those,
    whose exponentials relative to the largest score are below what fp16 holds. The bound: a rounding
    of the output and one of the large exponentials, 2^-11 each; the small ones' half spacing, 2^-32 of
    the sum's largest term, of which there are four; 2^-16 for 32-bit arithmetic."""
    heads, d, page, keys = 256, 64, 4096, 1 << 18
    lead, rest = 17.5, math.exp(-17.5)
    k = torch.zeros(2, page, heads, d, dtype=F16)
    v = torch.ones(2, page, heads, d, dtype=F16)
    k[0, 0:128:32, :, 0], v[0, 0:128:32] = lead, -1.0
    table = torch.ones(1, keys // page, dtype=torch.int32)
    table[0, 0] = 0
    q = torch.zeros(n, heads, d, dtype=F16)
    q[:, :, 0] = 1.0
    say("prefix_attention small weights", n)
    out, lse = g.prefix_attention(q.cuda(), k.cuda(), v.cuda(), i32([0, n]).cuda(), table.cuda(), i32([keys]).cuda(),
                                  scale=1.0, want_lse=True)
    torch.cuda.synchronize()
    seen = torch.arange(keys - n + 1, keys + 1, dtype=torch.float64)
    total = 4 + (seen - 4) * rest
    want = ((seen - 4) * rest - 4) / total
    off = float((out.cpu().double() - want[:, None, None]).abs().max())
    assert off <= 2.0 ** -10 + keys / 4 * 2.0 ** -32 + 2.0 ** -16
    assert float((lse.cpu().double() - lead - total.log()[:, None]).abs().max()) <= 2.0 ** -18 * 40


def test_gradients_are_refused_and_not_dropped():
    c = Case([1, 1], [5, 6], [(0, 2, 7)], 4, 2, 64, 16, F16)
    a = {**c.arguments(), "out": torch.zeros(2, 4, 64, dtype=F16, device="cuda"),
         "lse": torch.zeros(2, 4, device="cuda")}
    say("prefix_attention gradients")
    for name in ("q", "k_pages", "v_pages", "out", "lse"):
        b = {**a, name: a[name].clone().requires_grad_()}
        with pytest.raises(ValueError, match=name + " requires a gradient"):
            g.prefix_attention(**b)
        with torch.no_grad():
            g.prefix_attention(**b)
    with torch.autograd.forward_ad.dual_level():
        b = {**a, "q": torch.autograd.forward_ad.make_dual(a["q"], torch.ones_like(a["q"]))}
        with pytest.raises(ValueError, match="q requires a gradient"):
            g.prefix_attention(**b)


def test_thousands_of_sequences_and_groups():
    """Above 4,096 sequences and groups the plan keeps their offsets in the workspace, and with more
    rows than 2,048 workgroups join at once those go on to others."""
    gen = torch.Generator().manual_seed(11)
    groups, at = [], 0
    while len(groups) < 4200:
        end = at + 1 + (len(groups) % 7 == 0)
        groups.append((at, end, len(groups) % 23))
        at = end
    n_seq = at + 50
    own = torch.randint(0, 20, (n_seq,), generator=gen).tolist()
    n = torch.randint(0, 3, (n_seq,), generator=gen).tolist()
    c = Case(n, own, groups, 2, 1, 256, 16, F16)
    assert n_seq > 4096 and c.q.shape[0] * 2 > 2048 * 4  # 4 rows of 256 dims a workgroup
    c.check()


@pytest.mark.parametrize("n_seq,groups", [(62, 1), (64, 1), (65, 0), (200, 12), (1000, 23), (1023, 0), (1024, 1)])
def test_batches_on_both_sides_of_a_plan_of_their_own(n_seq, groups):
    gen = torch.Generator().manual_seed(n_seq)
    own = torch.randint(0, 90, (n_seq,), generator=gen).tolist()
    n = [1 + (i % 11 == 3) for i in range(n_seq)]
    n[5], own[5] = 70, 150
    first = [n_seq * i // max(groups, 1) for i in range(groups + 1)]
    Case(n, own, [(a, b, 17 + 40 * i) for i, (a, b) in enumerate(zip(first, first[1:]))], 4, 2, 64, 16, BF16,
         seed=n_seq).check()


@pytest.mark.parametrize("d,hkv", [(64, 64), (128, 32), (256, 16)])
def test_histories_that_are_not_kept_in_the_caches(d, hkv):
    """Of 128 MiB and a little, its end ragged and a page missing; three of the heads."""
    page, own = 16, 8203
    say("prefix_attention long history", d, hkv, own)
    gen = torch.Generator(device="cuda").manual_seed(d)
    pages = -(-own // page)
    kp, vp = (torch.randn(pages, hkv, page, d, generator=gen, device="cuda").to(BF16).transpose(1, 2) for _ in range(2))
    table = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)[None]
    table[0, 100] = -1
    q = torch.randn(1, hkv, d, generator=gen, device="cuda").to(BF16)
    first, length = i32([0, 1]), i32([own])
    assert own * hkv * 4 * d >= 128 << 20
    out, lse = g.prefix_attention(q, kp, vp, first.cuda(), table, length.cuda(), want_lse=True)
    torch.cuda.synchronize()
    for h in (0, hkv // 2 + 1, hkv - 1):
        o, l, o_tol, l_tol = R.attention(q[:, h:h + 1].cpu(), kp[:, :, h:h + 1].cpu(), vp[:, :, h:h + 1].cpu(), first,
                                         table.cpu(), length)
        R.near(lse[:, h:h + 1], l, l_tol, "lse")
        R.near(out[:, h:h + 1], o, o_tol, "out")


def test_a_cache_without_pages():
    say("prefix_attention without pages")
    none = torch.empty(0, 16, 2, 64, dtype=F16, device="cuda")
    q = torch.randn(3, 4, 64, device="cuda").to(F16)
    out, lse = g.prefix_attention(q, none, none, i32([0, 2, 3]).cuda(), i32([[0], [5]]).cuda(), i32([7, 1]).cuda(),
                                  i32([0, 2]).cuda(), i32([[0]]).cuda(), i32([9]).cuda(), want_lse=True)
    torch.cuda.synchronize()
    assert (out == 0).all() and (lse == -math.inf).all()
