"""kv_weigh and kv_evict on the GPU against plain computations on the CPU, and a run of all the paged cache's
calls together."""

import math

import pytest
import torch

import budget_reference as B
import kv_reference as R
import paper_2607_23115_amd as g
from gpu_util import say
from test_gpu_prefix_attention import Case

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    torch.cuda.init()


def i32(x):
    return torch.tensor(x, dtype=torch.int32)


def bits(x):
    x = x.detach().cpu().contiguous()
    return x.view(torch.int16 if x.element_size() == 2 else torch.int32)


class Weighed(Case):
    """A ragged batch with weights and births of every place, those that nobody may read NaN or -9."""

    def __init__(self, n, own, hq, hkv, d, page, dtype, seed=0, **kw):
        super().__init__(n, own, [], hq, hkv, d, page, dtype, seed=seed, **kw)
        gen = torch.Generator().manual_seed(seed + 100)
        self.weights = torch.full((self.kp.shape[0], hkv, page), math.nan)
        self.born = torch.full(self.weights.shape, -9, dtype=torch.int32)
        for s, (k, m) in enumerate(zip(n, own)):
            for j, (p, i) in enumerate(B.places(self.own_pages[s], m, page)):
                if j < m - k:
                    self.weights[p, :, i] = torch.rand(hkv, generator=gen) * 3
                    self.born[p, :, i] = j
        self.positions = torch.randint(0, 9999, (self.q.shape[0],), generator=gen, dtype=torch.int32)
        self.lse = torch.randn(self.q.shape[:2], generator=gen) * 2 + math.log(1 + max(own))

    def call(self, a=None, **more):
        a = a or self.arguments()
        weights, born = self.weights.cuda(), self.born.cuda()
        out = more.pop("weights_out", None)
        got = g.kv_weigh(a["q"], a["k_pages"], a["q_first"], a["own_pages"], a["own_len"], self.lse.cuda(), weights,
                         born=born, positions=self.positions.cuda(), scale=self.scale, weights_out=out, **more)
        torch.cuda.synchronize()
        assert got is (weights if out is None else out)
        return got, born

    def want(self):
        return B.weigh(self.q, self.kp, self.q_first, self.own_pages, self.own_len, self.lse, self.weights, self.born,
                       self.positions, self.scale)

    def check(self, a=None, **more):
        say("kv_weigh", self.what)
        got, born = self.call(a, **more)
        want, births, tol = self.want()
        assert torch.equal(born.cpu(), births)
        R.near(got, want, tol, "weights")
        return got


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_types_and_widths(dtype, d):
    Weighed([1, 1, 1], [1, 70, 300], 8, 2, d, 16, dtype).check()
    Weighed([5, 40, 9], [5, 60, 300], 4, 2, d, 32, dtype).check()
    Weighed([150, 33], [150, 50], 2, 1, d, 16, dtype).check()


@pytest.mark.parametrize("hq,hkv", [(1, 1), (5, 5), (3, 1), (7, 1), (28, 4), (32, 32), (24, 8), (40, 2), (17, 1)])
def test_heads(hq, hkv):
    Weighed([1, 3, 1], [40, 33, 1], hq, hkv, 64, 16, BF16, seed=hq).check()
    Weighed([50], [50], hq, hkv, 64, 16, F16, seed=hq).check()


@pytest.mark.parametrize("own", [1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 1000, 5001])
def test_one_token_of_one_sequence(own):
    Weighed([1], [own], 4, 1, 128, 16, BF16, seed=own).check()


@pytest.mark.parametrize("n,own", [(16, 16), (28, 28), (29, 29), (32, 200), (64, 64), (65, 65), (127, 130), (200, 333),
                                   (300, 300), (130, 129)])
def test_prompts(n, own):
    """Tokens on both sides of where waves start to share keys (8 tiles of 16 rows)."""
    Weighed([n], [own], 4, 1, 64, 16, BF16, seed=n).check()
    Weighed([n, 1, n // 2], [own, 77, n // 2], 3, 1, 128, 64, F16, seed=n).check()


@pytest.mark.parametrize("dtype,d", [(F16, 64), (BF16, 128), (F16, 256)])
def test_new_tokens_of_many_sequences(dtype, d):
    """3 to 14 tiles of rows each, with as many sequences and heads as there are CUs, and with one fewer."""
    n = [12 + i % 44 for i in range(128)]
    Weighed(n, [m + 11 * i % 150 for i, m in enumerate(n)], 8, 2, d, 16, dtype, seed=d).check()
    Weighed(n[:85], [m + 13 * i % 70 for i, m in enumerate(n[:85])], 12, 3, d, 16, dtype, seed=d).check()


@pytest.mark.parametrize("page,head_major", [(16, False), (64, True), (256, False), (4096, True)])
def test_pages(page, head_major):
    Weighed([1, 2], [page + 1, 2 * page - 1], 4, 2, 64, page, F16, head_major=head_major).check()


def test_sequences_without_tokens_keys_or_either():
    """A sequence without tokens keeps its weights; one with more tokens than keys; tokens of no sequence."""
    Weighed([4, 3, 0, 6, 0], [2, 0, 50, 6, 0], 4, 2, 64, 16, F16, pad_tokens=5).check()
    c = Weighed([0, 0], [30, 40], 4, 2, 64, 16, F16)
    out = torch.full(c.weights.shape, 5.0, device="cuda")
    got, _ = c.call(weights_out=out)
    want = c.weights.clone()
    want[torch.isnan(want)] = 5.0
    assert torch.equal(got.cpu(), want)


def test_weights_that_go_elsewhere():
    """Only the places of own keys are written."""
    c = Weighed([2, 30], [40, 90], 4, 2, 64, 16, BF16)
    want, _, tol = c.want()
    out = torch.full(c.weights.shape, -5.0, device="cuda")
    got, _ = c.call(weights_out=out)
    mine = ~torch.isnan(want)
    R.near(got[mine.cuda()], want[mine], tol[mine], "weights")
    assert (got.cpu()[~mine] == -5).all()


def test_rows_that_are_left_out_and_strided_queries():
    c = Weighed([3, 40], [40, 90], 4, 2, 64, 16, BF16)
    c.lse[1], c.lse[20:30, 2] = math.inf, math.inf
    c.scale = -0.3
    wide = torch.randn(c.q.shape[0], 9, 64).to(BF16)
    wide[:, 2:6] = c.q
    c.check({**c.arguments(), "q": wide.cuda()[:, 2:6]})


@pytest.mark.parametrize("dtype,d", [(F16, 64), (BF16, 128), (BF16, 256)])
@pytest.mark.parametrize("n", [1, 5, 20, 40, 56, 57, 140, 300])
def test_rows_that_are_left_out_may_hold_anything(n, dtype, d):
    """Queries of rows whose lse is +infinity, as padded ones have that nobody wrote: NaN, infinite, or so large that
    their scores overflow. 1 to 7 tiles of rows that are few, and many, whose last tiles see all of a block's keys."""
    c = Weighed([n, 3], [n + 90, 40], 4, 2, d, 16, dtype, seed=n)
    anything = (math.nan, math.inf, -math.inf, torch.finfo(dtype).max)
    rows = [(t, h, anything[i % 4]) for i, (t, h) in enumerate((t, h) for t in {0, n // 2, n - 1, n + 1} for h in range(4)
                                                               if t != n // 2 or h in (0, 3))]
    for t, h, _ in rows:
        c.lse[t, h] = math.inf
    want, births, tol = c.want()  # of finite queries, whose rows add exp(-infinity) = 0
    for t, h, x in rows:
        c.q[t, h] = x
        c.q[t, h, ::3] *= -1
    say("kv_weigh", c.what)
    got, born = c.call()
    assert torch.equal(born.cpu(), births)
    R.near(got, want, tol, "weights")


@pytest.mark.parametrize("n", [5, 140])
def test_what_a_row_does_not_see_may_be_anything(n):
    """NaN in a late key reaches that key's weight alone, NaN in a query what the query sees."""
    c = Weighed([n], [n + 40], 4, 2, 64, 16, BF16)
    p, i = B.places(c.own_pages[0], n + 40, 16)[n + 38]
    c.kp[p, i, 1] = math.nan
    c.q[n - 3, 0] = math.nan  # key head 0
    got, _ = c.call()
    want, _, tol = c.want()
    got = got.cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    fine = torch.isfinite(want)
    assert bool(((got - want).abs()[fine] <= tol[fine]).all())


def test_missing_pages_and_lengths_out_of_range():
    c = Weighed([1, 2, 100], [100, 60, 130], 4, 2, 64, 16, F16)
    c.own_pages[0, 2], c.own_pages[1, 0], c.own_pages[2, 5] = -1, c.kp.shape[0], 1 << 30
    c.check()
    c = Weighed([1, 1, 2], [32, 20, 20], 2, 1, 64, 16, F16)
    a = c.arguments()
    a["own_pages"] = a["own_pages"][:, :2].contiguous()
    say("kv_weigh lengths out of range")
    a["k_pages"][torch.isnan(a["k_pages"])] = 0.5
    for name, odd, same in (("own_len", [1 << 30, -5, 20], [32, 0, 20]), ("q_first", [-3, 1, 2, 99], [0, 1, 2, 4])):
        x, y = (c.call({**a, name: i32(v).cuda()}) for v in (odd, same))
        assert torch.equal(bits(x[0]), bits(y[0])) and torch.equal(x[1], y[1])


def test_many_sequences():
    gen = torch.Generator().manual_seed(4)
    own = torch.randint(0, 40, (700,), generator=gen).tolist()
    n = torch.randint(0, 3, (700,), generator=gen).tolist()
    n[50], own[50], n[300], own[300] = 90, 200, 1, 900
    Weighed(n, own, 2, 1, 64, 16, F16).check()


class Streamed:
    """Long sequences, made and weighed on the GPU: the plain computation in 64 bits takes all keys of a sequence and
    head at once. Units of work are halves of 64 keys of each sequence and head, dealt out evenly to 2,048 waves (1,024
    of heads of 256)."""

    def __init__(self, n, own, hq, hkv, d, page, dtype, seed=0):
        gen = torch.Generator("cuda").manual_seed(seed)
        self.n, self.own, self.hkv, self.d, self.page = n, own, hkv, d, page
        counts = [-(-m // page) for m in own]
        order = torch.randperm(sum(counts) + 1, generator=gen, device="cuda")
        self.kp = torch.randn(sum(counts) + 1, page, hkv, d, generator=gen, device="cuda", dtype=dtype)
        table = torch.full((len(own), max(counts) + 1), -1, dtype=torch.int32, device="cuda")
        self.pages, at = [], 0
        for s, count in enumerate(counts):
            self.pages.append(order[at:at + count])
            table[s, :count] = self.pages[-1].int()
            at += count
        self.q = torch.randn(sum(n), hq, d, generator=gen, device="cuda", dtype=dtype)
        self.lse = torch.randn(sum(n), hq, generator=gen, device="cuda") * 2 + math.log(max(own))
        self.weights = torch.rand(self.kp.shape[0], hkv, page, generator=gen, device="cuda") * 3
        self.born = torch.randint(0, 999, self.weights.shape, generator=gen, device="cuda", dtype=torch.int32)
        self.positions = torch.randint(1000, 9999, (sum(n),), generator=gen, device="cuda", dtype=torch.int32)
        self.q_first, self.table, self.own_len = (x.cuda() for x in (i32([sum(n[:i]) for i in range(len(n) + 1)]), table,
                                                                     i32(own)))

    def halves(self):
        return sum(-(-m // 32) for m in self.own) * self.hkv

    def want(self):
        """(weights, born, bound), the bound being B.weigh's."""
        out, births, tol = self.weights.double(), self.born.clone(), torch.zeros_like(self.weights, dtype=torch.float64)
        ratio, scale = self.q.shape[1] // self.hkv, self.d ** -0.5
        t0 = 0
        for n, own, pages in zip(self.n, self.own, self.pages):
            j = torch.arange(own, device="cuda")
            p, i = pages[j // self.page], j % self.page
            for h in range(self.hkv):
                k = self.kp[p, i, h].double()
                total = torch.where(j < own - n, out[p, h, i], 0.0)
                bound = torch.zeros(own, dtype=torch.float64, device="cuda")
                for t in range(n):
                    for r in range(h * ratio, (h + 1) * ratio):
                        x, l = self.q[t0 + t, r].double(), self.lse[t0 + t, r].double()
                        score, size = (k * x).sum(-1) * scale, (k * x).abs().sum(-1) * scale
                        e = torch.where(j < own - n + t + 1, torch.exp(score - l), 0.0)
                        total = total + e
                        bound += 2 * e * ((self.d + 4) * 2.0 ** -24 * size + 2.0 ** -22 * (1 + score.abs() + l.abs()))
                out[p, h, i] = total
                tol[p, h, i] = bound + (n * ratio / 16 + 12) * 2.0 ** -24 * total.abs() + 2.0 ** -120
                births[p[own - n:], h, i[own - n:]] = self.positions[t0:t0 + n]
            t0 += n
        return out, births, tol

    def call(self):
        weights, born = self.weights.clone(), self.born.clone()
        g.kv_weigh(self.q, self.kp, self.q_first, self.table, self.own_len, self.lse, weights, born, self.positions)
        torch.cuda.synchronize()
        return weights, born

    def check(self):
        say("kv_weigh", f"n={self.n} own={self.own} heads={self.q.shape[1]}/{self.hkv} d={self.d} page={self.page}",
            self.kp.dtype)
        got, born = self.call()
        want, births, tol = self.want()
        assert torch.equal(born, births)
        R.near(got, want.cpu(), tol.cpu(), "weights")
        again, _ = self.call()
        assert torch.equal(got, again)


def test_the_plain_sums_of_long_sequences():
    """The computation that takes all keys at once is the one that takes one at a time."""
    c = Streamed([2, 1, 9], [40, 17, 70], 4, 2, 64, 16, BF16)
    want, births, tol = (x.cpu() for x in c.want())
    one, born, bound = B.weigh(*(x.cpu() for x in (c.q, c.kp, c.q_first, c.table, c.own_len, c.lse, c.weights, c.born,
                                                   c.positions)))
    assert torch.equal(births, born) and float((want - one).abs().max()) < 1e-12
    assert float((tol - bound).abs().max()) < 1e-12
    c.check()


@pytest.mark.parametrize("dtype,d", [(F16, 64), (BF16, 128), (BF16, 256)])
@pytest.mark.parametrize("n", [[1, 1, 1, 2, 1, 3], [9, 4, 12, 8, 10, 12], [20, 28, 13, 25, 18, 24]])
def test_waves_that_go_from_one_head_and_sequence_to_the_next(n, dtype, d):
    """One tile of rows, two and three (which stay in LDS), and 4 to 7 (loaded again); several halves a wave."""
    c = Streamed(n, [60001, n[1], 90000, 26000, 777, 58000], 8, 2, d, 16, dtype, seed=d)
    assert c.halves() > 7 * 2048 and c.halves() % 2048
    c.check()


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F16, 128), (BF16, 256)])
def test_many_sequences_of_several_halves_a_wave(dtype, d):
    """More sequences than are looked at in one step, some of them with rows for a workgroup (15 tiles)."""
    n = [60 if i in (3, 70, 149) else 1 + i % 3 for i in range(150)]
    c = Streamed(n, [m + 97 * i % 5000 for i, m in enumerate(n)], 8, 2, d, 32, dtype, seed=d)
    assert c.halves() > 10 * 2048
    c.check()


@pytest.mark.parametrize("dtype,d,own", [(BF16, 64, 2_400_017), (F16, 128, 2_400_017), (BF16, 256, 1_200_017)])
@pytest.mark.parametrize("n", [1, 11])
def test_waves_that_look_up_pages_again(n, dtype, d, own):
    """More than 32 halves a wave: pages are looked up for 32 at a time."""
    c = Streamed([n], [own], 4, 1, d, 64, dtype, seed=n)
    assert c.halves() > 36 * (1024 if d == 256 else 2048)
    c.check()


def test_twice_on_a_stream_and_in_a_graph():
    c = Weighed([1, 60, 1], [900, 300, 44], 8, 2, 128, 16, BF16)
    a = c.arguments()
    a["k_pages"][torch.isnan(a["k_pages"])] = 0.5
    first, born = c.call(a)
    side = torch.cuda.Stream()
    say("kv_weigh stream and graph")
    again, _ = c.call(a, stream=side)
    side.synchronize()
    assert torch.equal(bits(first), bits(again))
    weights, lse, pos = c.weights.cuda(), c.lse.cuda(), c.positions.cuda()
    births, out = c.born.cuda(), torch.empty_like(weights)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g.kv_weigh(a["q"], a["k_pages"], a["q_first"], a["own_pages"], a["own_len"], lse, weights, births, pos, out)
    for own in ([900, 300, 44], [13, 70, 0], [901, 304, 48]):
        a["own_len"].copy_(i32(own))
        out.zero_()
        want = torch.zeros_like(out)
        g.kv_weigh(a["q"], a["k_pages"], a["q_first"], a["own_pages"], a["own_len"], lse, weights, births.clone(), pos, want)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(want))


def test_the_weights_of_a_query_add_up_to_one():
    """With the lse that attention returned, a row's weights sum to 1: all of a head's to its rows."""
    c = Weighed([3, 100], [300, 400], 8, 2, 128, 16, BF16)
    a = c.arguments()
    _, lse = g.prefix_attention(**a, want_lse=True)
    out = torch.zeros(c.weights.shape, device="cuda")
    g.kv_weigh(a["q"], a["k_pages"], a["q_first"], a["own_pages"], a["own_len"], lse, torch.zeros_like(out),
               weights_out=out)
    sums = out.sum((0, 2)).cpu()
    # 412 rows a head, each off by at most what its scores, its lse and 32-bit sums are: 2^-12
    assert float((sums - 103 * 4).abs().max()) <= 412 * 2.0 ** -12


def test_weigh_refusals():
    c = Weighed([1, 1], [5, 6], 4, 2, 64, 16, F16)
    a = c.arguments()
    w, b, lse, pos = torch.full(c.weights.shape, 3.0, device="cuda"), c.born.cuda(), c.lse.cuda(), c.positions.cuda()
    good = dict(q=a["q"], k_pages=a["k_pages"], q_first=a["q_first"], own_pages=a["own_pages"], own_len=a["own_len"],
                lse=lse, weights=w, born=b, positions=pos)
    for message, bad in (("q must be", {"q": a["q"].float()}), ("multiple of kv_heads", {"q": a["q"][:, :3].contiguous(), "lse": lse[:, :3].contiguous()}),
                         ("lse must be", {"lse": lse[:1]}), ("lse must be", {"lse": lse.half()}),
                         ("weights must be", {"weights": w[:1]}), ("weights must be", {"weights": w.double()}),
                         ("born must be", {"born": b[:, :1]}), ("born is required", {"born": None}),
                         ("positions is required", {"positions": None}), ("positions holds", {"positions": pos[:1]}),
                         ("q_first holds 2", {"q_first": a["q_first"][:2]}), ("own_pages must be", {"own_pages": a["own_pages"][:1]}),
                         ("on the GPU", {"k_pages": a["k_pages"].cpu()})):
        with pytest.raises((ValueError, g.GleamError), match=message):
            g.kv_weigh(**{**good, **bad})
    flat = torch.zeros(w.numel() + 8, device="cuda")
    with pytest.raises(g.GleamError, match="not overlap"):
        g.kv_weigh(**{**good, "weights": flat[:-8].view(w.shape), "weights_out": flat[8:].view(w.shape)})
    for name in ("q", "k_pages", "lse", "weights"):
        with pytest.raises(ValueError, match=name + " requires a gradient"):
            g.kv_weigh(**{**good, name: good[name].clone().requires_grad_()})
    torch.cuda.synchronize()
    assert (w == 3).all()


# --------------------------------------------------------------------------- #
class Evicted:
    """Sequences of `own` keys each. kind: how weights are drawn."""

    def __init__(self, own, hkv, d, page, dtype, keep, sinks=0, recent=0, kind="random", seed=0, head_major=True):
        gen = torch.Generator().manual_seed(seed)
        c = Case([0] * len(own), own, [], hkv, hkv, d, page, dtype, seed=seed)
        self.kp, self.vp, self.own_pages, self.own_len = c.kp, c.vp, c.own_pages, c.own_len
        self.weights = torch.full((self.kp.shape[0], hkv, page), math.nan)
        self.born = torch.full(self.weights.shape, -9, dtype=torch.int32)
        for s, m in enumerate(own):
            order = torch.stack([torch.randperm(m, generator=gen) for _ in range(hkv)]) if m else None
            for j, (p, i) in enumerate(B.places(self.own_pages[s], m, page)):
                w = torch.randn(hkv, generator=gen)
                if kind == "few":
                    w = (w * 2).round()
                elif kind == "same":
                    w = torch.zeros(hkv)
                elif kind == "odd":
                    pick = torch.randint(0, 6, (hkv,), generator=gen)
                    w = torch.where(pick == 0, torch.tensor(math.nan), w)
                    w = torch.where(pick == 1, torch.tensor(math.inf), w)
                    w = torch.where(pick == 2, torch.tensor(-math.inf), w)
                    w = torch.where(pick == 3, torch.where(torch.rand(hkv, generator=gen) < 0.5, 0.0, -0.0), w)
                self.weights[p, :, i], self.born[p, :, i] = w, order[:, j].to(torch.int32)
        self.total = self.own_len.clone()
        self.keep, self.sinks, self.recent, self.head_major = keep, sinks, recent, head_major
        self.what = f"own={own if len(own) < 9 else len(own)} heads={hkv} d={d} page={page} {dtype} keep={keep} {kind}"

    def arguments(self):
        def pages(t):
            return t.transpose(1, 2).contiguous().cuda().transpose(1, 2) if self.head_major else t.cuda()
        return dict(k_pages=pages(self.kp), v_pages=pages(self.vp), own_pages=self.own_pages.cuda(),
                    own_len=self.own_len.cuda(), weights=self.weights.cuda(), born=self.born.cuda(),
                    total=self.total.cuda(), keep=self.keep, sinks=self.sinks, recent=self.recent)

    def want(self):
        return B.evict(self.kp, self.vp, self.own_pages, self.own_len, self.weights, self.born, self.total, self.keep,
                       self.sinks, self.recent)

    def check(self):
        """In place, and with weights and births that go elsewhere."""
        say("kv_evict", self.what)
        want = self.want()
        a = self.arguments()
        length = g.kv_evict(**a)
        torch.cuda.synchronize()
        for x, y, name in zip((a["k_pages"], a["v_pages"], a["weights"], a["born"], length), want,
                              ("keys", "values", "weights", "born", "len_out")):
            assert torch.equal(bits(x), bits(y)), name
        a = self.arguments()
        w, b = torch.full_like(a["weights"], 7.0), torch.full_like(a["born"], 7)
        out = torch.empty_like(a["own_len"])
        assert g.kv_evict(**a, weights_out=w, born_out=b, len_out=out) is out
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), want[4]) and torch.equal(bits(a["k_pages"]), bits(want[0]))
        assert torch.equal(bits(a["weights"]), bits(self.weights)) and torch.equal(bits(a["born"]), bits(self.born))
        page, mine = self.kp.shape[1], torch.zeros(self.weights.shape, dtype=torch.bool)
        for s, m in enumerate(want[4].tolist()):
            for p, i in B.places(self.own_pages[s], m, page):
                if 0 <= p < self.kp.shape[0]:
                    mine[p, :, i] = True
        assert torch.equal(bits(w.cpu()[mine]), bits(want[2][mine])) and (w.cpu()[~mine] == 7).all()
        assert torch.equal(b.cpu()[mine], want[3][mine]) and (b.cpu()[~mine] == 7).all()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_evicting(dtype, d):
    Evicted([0, 1, 40, 63, 64, 65, 100, 300], 2, d, 16, dtype, 64, seed=d).check()
    Evicted([90, 7, 200], 3, d, 32, dtype, 30, sinks=2, recent=9, head_major=False).check()


@pytest.mark.parametrize("kind", ["random", "few", "same", "odd"])
@pytest.mark.parametrize("keep", [0, 1, 17, 99, 100, 101])
def test_kinds_of_weights(kind, keep):
    """Ties, weights that are all the same, NaN, infinities and zeros of both signs; budgets of nothing, one,
    all but one and all."""
    Evicted([100, 101, 163], 2, 64, 16, F16, keep, sinks=keep % 3, recent=keep // 4, kind=kind).check()


def test_more_to_keep_than_the_budget():
    """Protected keys alone are over the budget: the first places of them stay."""
    Evicted([100, 150], 2, 64, 16, F16, 20, sinks=15, recent=40).check()
    Evicted([100, 150], 2, 64, 16, F16, 20, sinks=1 << 31, recent=0).check()
    Evicted([100, 150], 2, 64, 16, F16, 20, sinks=0, recent=(1 << 32) - 1).check()
    c = Evicted([100, 150], 2, 64, 16, F16, 20, recent=10)
    c.total += 1000  # none of the last ten is in the cache any more
    c.check()


@pytest.mark.parametrize("own,keep", [(255, 100), (257, 256), (1023, 512), (1025, 1000), (2050, 2048), (4000, 1500),
                                      (4070, 2001), (4500, 700), (20000, 9000), (40000, 300), (33000, 32000)])
def test_long_sequences(own, keep):
    """On both sides of what a workgroup's registers hold, for narrow tables and for wide ones."""
    Evicted([own], 1, 64, 16, F16, keep, sinks=4, recent=keep // 8, kind="few" if own % 2 else "random").check()


@pytest.mark.parametrize("d", [64, 128, 256])
def test_many_sequences_and_heads_of_narrow_tables(d):
    """Whose workgroups copy the pairs themselves."""
    Evicted([600 + 7 * i for i in range(16)], 8, d, 16, BF16, 400, recent=30, kind="few", seed=d).check()
    Evicted([4000, 3100, 1, 0, 2049, 2047, 4064, 2500], 16, d, 32, F16, 2048, sinks=3, recent=100).check()


@pytest.mark.parametrize("own,keep", [(100, 90), (5000, 4990), (40000, 39990)])
def test_missing_pages_go_before_nan(own, keep):
    """Ten keys of 16 in a page that is none go, and none of the NaN weights in the page behind it."""
    c = Evicted([own], 2, 64, 16, F16, keep)
    gone, behind = int(c.own_pages[0, 1]), int(c.own_pages[0, 2])
    c.weights[gone], c.born[gone] = math.nan, -9
    c.weights[behind] = math.nan
    c.own_pages[0, 1] = -1
    before = c.kp.clone()
    c.check()
    assert torch.equal(bits(c.want()[0][behind]), bits(before[behind]))


def test_missing_pages():
    c = Evicted([100, 90], 2, 64, 16, F16, 40, recent=5)
    c.own_pages[0, 1], c.own_pages[0, 5], c.own_pages[1, 3] = -1, c.kp.shape[0], 1 << 30
    c.check()


def test_many_sequences_are_evicted():
    Evicted([20 + i % 40 for i in range(1200)], 2, 64, 16, F16, 32, recent=3).check()


def test_evict_streams_graphs_and_lengths_out_of_range():
    c = Evicted([300, 500, 40], 2, 128, 16, BF16, 200, sinks=4, recent=50)
    a, want = c.arguments(), c.want()
    say("kv_evict stream and graph")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    length = g.kv_evict(**a, stream=side)
    side.synchronize()
    for x, y in zip((a["k_pages"], a["v_pages"], a["weights"], a["born"], length), want):
        assert torch.equal(bits(x), bits(y))
    a, kept = c.arguments(), c.arguments()
    out, ws = torch.empty_like(a["own_len"]), g.kv_evict_workspace(a["k_pages"], a["v_pages"], 3, a["own_pages"].shape[1], 200)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        g.kv_evict(**a, len_out=out, ws=ws)
    for own in ([300, 500, 40], [250, 201, 30], [300, 500, 1]):
        for name in ("k_pages", "v_pages", "weights", "born"):
            a[name].copy_(kept[name])
        a["own_len"].copy_(i32(own))
        c.own_len = i32(own)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((a["k_pages"], a["v_pages"], a["weights"], a["born"], out), c.want()):
            assert torch.equal(bits(x), bits(y))
        ws.fill_(255)
        out.zero_()
    a = kept
    say("kv_evict lengths out of range")
    a["own_len"].copy_(i32([-4, 1 << 30, 3]))
    a["own_pages"] = a["own_pages"][:, :10].contiguous()
    assert g.kv_evict(**{**a, "keep": 100}).tolist() == [0, 100, 3]


def test_evict_refusals():
    c = Evicted([50, 60], 2, 64, 16, F16, 20)
    a = c.arguments()
    for message, bad in (("weights must be", {"weights": a["weights"][:1]}), ("born must be", {"born": a["born"].long()}),
                         ("total holds", {"total": a["total"][:1]}), ("own_len must be", {"own_len": a["own_len"].long()}),
                         ("own_pages must be", {"own_pages": a["own_pages"][:1]}), ("keep must not", {"keep": -1}),
                         ("recent must not", {"recent": 1 << 32}),
                         ("workspace of 256 bytes", {"ws": torch.empty(256, dtype=torch.uint8, device="cuda")}),
                         ("overlap", {"k_pages": a["k_pages"][:, :, :1].expand(-1, -1, 2, -1)}),
                         ("differ in shape", {"v_pages": a["v_pages"][:1]}),
                         ("len_out holds", {"len_out": a["own_len"][:1]}), ("overlap own_len", {"len_out": a["own_len"]})):
        with pytest.raises((ValueError, g.GleamError), match=message):
            g.kv_evict(**{**a, **bad})
    for name in ("k_pages", "v_pages", "weights"):
        with pytest.raises(ValueError, match=name + " requires a gradient"):
            g.kv_evict(**{**a, name: a[name].clone().requires_grad_()})
    torch.cuda.synchronize()
    for name, x in (("k_pages", c.kp), ("weights", c.weights), ("born", c.born)):
        assert torch.equal(bits(a[name]), bits(x))


def test_caches_without_pages_or_sequences():
    none = torch.empty(0, 16, 2, 64, dtype=F16, device="cuda")
    w, b = torch.empty(0, 2, 16, device="cuda"), torch.empty(0, 2, 16, dtype=torch.int32, device="cuda")
    q, lse = torch.randn(3, 4, 64, device="cuda").to(F16), torch.zeros(3, 4, device="cuda")
    first, table, own = i32([0, 2, 3]).cuda(), i32([[0], [5]]).cuda(), i32([7, 1]).cuda()
    say("budget calls without pages")
    assert g.kv_weigh(q, none, first, table, own, lse, w, b, i32([1, 2, 3]).cuda()) is w
    assert g.kv_evict(none, none, table, own, w, b, own, 4).tolist() == [0, 0]
    seen = torch.full((3, 1), -1, dtype=torch.int64, device="cuda")
    assert g.kv_accept(none, none, first, seen, i32([1, 0]).cuda(), table, own).tolist() == [0, 0]
    out, _ = g.tree_attention(q, none, none, first, seen, table, own)
    assert (out == 0).all()
    page = torch.zeros(2, 16, 2, 64, dtype=F16, device="cuda")
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    nobody = torch.empty(0, 3, dtype=torch.int32, device="cuda")
    w, b = torch.zeros(2, 2, 16, device="cuda"), torch.zeros(2, 2, 16, dtype=torch.int32, device="cuda")
    assert g.kv_evict(page, page, nobody, empty, w, b, empty, 4).numel() == 0
    assert g.kv_accept(page, page, i32([0]).cuda(), seen, empty, nobody, empty).numel() == 0
    g.kv_weigh(q, page, i32([0]).cuda(), nobody, empty, lse, w, b, i32([1, 2, 3]).cuda())
    torch.cuda.synchronize()


def test_a_cache_beyond_32_bit_offsets():
    """Keys, weights and births of the last page, past 2^32 elements of the cache."""
    page, d = 4096, 128
    pages = (1 << 32) // (page * d) + 3
    say("budget calls, large cache", pages)
    kp = torch.zeros(pages, page, 1, d, dtype=BF16, device="cuda")
    vp = torch.zeros_like(kp)
    gen = torch.Generator().manual_seed(0)
    k, v = (torch.randn(100, 1, d, generator=gen).to(BF16) for _ in range(2))
    kp[-1, :100], vp[-1, :100] = k.cuda(), v.cuda()
    w, b = torch.zeros(pages, 1, page, device="cuda"), torch.zeros(pages, 1, page, dtype=torch.int32, device="cuda")
    w[-1, 0, :100] = torch.rand(100, generator=gen).cuda()
    b[-1, 0, :100] = torch.arange(100, dtype=torch.int32, device="cuda")
    q, lse = torch.randn(1, 4, d, generator=gen).to(BF16), torch.randn(1, 4, generator=gen) + 5
    small = lambda x: x[-1:].cpu()  # noqa: E731
    first, table, own, at0 = i32([0, 1]), i32([[pages - 1]]), i32([100]), i32([[0]])
    want, births, tol = B.weigh(q, small(kp), first, at0, own, lse, small(w), small(b), i32([777]))
    g.kv_weigh(q.cuda(), kp, first.cuda(), table.cuda(), own.cuda(), lse.cuda(), w, b, i32([777]).cuda())
    assert torch.equal(small(b), births)
    R.near(small(w), want, tol, "weights")
    want = B.evict(small(kp), small(vp), at0, own, small(w), small(b), i32([778]), 30, 2, 5)
    out = g.kv_evict(kp, vp, table.cuda(), own.cuda(), w, b, i32([778]).cuda(), 30, 2, 5)
    for x, y in zip((small(kp), small(vp), small(w), small(b), out), want):
        assert torch.equal(bits(x), bits(y))
    seen = torch.tensor([[0b10010], [0b01010], [0], [0b11000], [0b10101]])
    n = i32([0, 5])
    kw, vw, lw = B.accept(small(kp), small(vp), n, seen, i32([4]), at0, i32([30]))
    lg = g.kv_accept(kp, vp, n.cuda(), seen.cuda(), i32([4]).cuda(), table.cuda(), i32([30]).cuda())
    assert torch.equal(lg.cpu(), lw) and torch.equal(bits(small(kp)), bits(kw)) and torch.equal(bits(small(vp)), bits(vw))


def test_a_run_of_them_together():
    """Two sequences served: prompts appended, attended to and weighed; a tree of drafts checked, one path of it
    accepted and weighed; the cache cut down to its budget; a next token behind what is left. After each
    step the cache holds what the plain computations say."""
    hq, hkv, d, page, dtype = 4, 2, 64, 16, BF16
    gen = torch.Generator().manual_seed(1)
    table = i32([[3, 7, 1, 9, 4, 0], [2, 8, 5, 6, 10, 11]])
    kp, vp = (torch.zeros(12, page, hkv, d, dtype=dtype) for _ in range(2))
    w, b = torch.full((12, hkv, page), 99.0), torch.full((12, hkv, page), -1, dtype=torch.int32)
    dk, dv, dw, db, dtable = kp.cuda(), vp.cuda(), w.cuda(), b.cuda(), table.cuda()
    rotary = g.rotary_table(256, d)

    def append(per_seq, at, positions):
        """New tokens of each sequence at places from at[s] on, at their positions."""
        n = sum(per_seq)
        q, k, v = (torch.randn(n, h, d, generator=gen).to(dtype) for h in (hq, hkv, hkv))
        slots = torch.tensor([int(table[s, j // page]) * page + j % page for s, m in enumerate(per_seq)
                              for j in range(at[s], at[s] + m)])
        out = g.kv_append(k.cuda(), v.cuda(), dk, dv, slots.cuda(), q=q.cuda(), positions=positions.cuda(), rotary=rotary)
        return out

    def weigh(q, first, own, lse, positions):
        want, births, tol = B.weigh(q.cpu(), dk.cpu(), first, table, own, lse.cpu(), dw.cpu(), db.cpu(), positions)
        g.kv_weigh(q, dk, first.cuda(), dtable, own.cuda(), lse, dw, db, positions.cuda())
        assert torch.equal(db.cpu(), births)
        R.near(dw, want, tol, "weights")

    # prompts
    n = [50, 30]
    first, own = i32([0, 50, 80]), i32(n)
    positions = torch.cat([torch.arange(m, dtype=torch.int32) for m in n])
    q = append(n, [0, 0], positions)
    out, lse = g.prefix_attention(q, dk, dv, first.cuda(), dtable, own.cuda(), want_lse=True)
    o, l, o_tol, l_tol = R.attention(q.cpu(), dk.cpu(), dv.cpu(), first, table, own)
    R.near(out, o, o_tol, "prompt")
    weigh(q, first, own, lse, positions)
    # drafts
    m = [7, 5]
    parent, first = i32([-1, 0, 0, 1, 1, 2, 4, -1, 0, 1, 0, 3]), i32([0, 7, 12])
    seen, depth = g.draft_tree(parent.cuda(), first.cuda(), 7)
    positions = depth.cpu() + torch.repeat_interleave(own, torch.tensor(m))
    q = append(m, n, positions)
    own = i32([57, 35])
    out, lse = g.tree_attention(q, dk, dv, first.cuda(), seen, dtable, own.cuda(), want_lse=True)
    o, l, o_tol, l_tol = B.tree_attention(q.cpu(), dk.cpu(), dv.cpu(), first, seen.cpu(), table, own)
    R.near(out, o, o_tol, "drafts")
    R.near(lse, l, l_tol, "lse")
    # the path 0, 1, 4, 6 of the first, 0, 3, 4 of the second, whose parents' indexes are 0, 0, 1, 0, 3
    leaf = i32([6, 4])
    kw, vw, lw = B.accept(dk.cpu(), dv.cpu(), first, seen.cpu(), leaf, table, own)
    own_out = g.kv_accept(dk, dv, first.cuda(), seen, leaf.cuda(), dtable, own.cuda())
    assert own_out.tolist() == lw.tolist() == [54, 33]
    assert torch.equal(bits(dk), bits(kw)) and torch.equal(bits(dv), bits(vw))
    path = torch.tensor([0, 1, 4, 6, 7, 10, 11])
    own, first = own_out.cpu(), i32([0, 4, 7])
    weigh(q[path.cuda()], first, own, lse[path.cuda()], positions[path])
    # down to 24 keys each
    total = i32([54, 33])
    want = B.evict(dk.cpu(), dv.cpu(), table, own, dw.cpu(), db.cpu(), total, 24, 2, 6)
    own_out = g.kv_evict(dk, dv, dtable, own.cuda(), dw, db, total.cuda(), 24, sinks=2, recent=6)
    for x, y in zip((dk, dv, dw, db, own_out), want):
        assert torch.equal(bits(x), bits(y))
    for s in range(2):
        for h in range(hkv):
            born = {int(db[p, h, i]) for p, i in B.places(table[s], 24, page)}
            assert len(born) == 24 and {0, 1} <= born and set(range(int(total[s]) - 6, int(total[s]))) <= born
    # one more token each
    first, own = i32([0, 1, 2]), i32([25, 25])
    q = append([1, 1], [24, 24], total)
    out, lse = g.prefix_attention(q, dk, dv, first.cuda(), dtable, own.cuda(), want_lse=True)
    o, l, o_tol, l_tol = R.attention(q.cpu(), dk.cpu(), dv.cpu(), first, table, own)
    R.near(out, o, o_tol, "next token")
    weigh(q, first, own, lse, total)
