"""kv_append and rotary_table on the GPU against 64-bit arithmetic on the CPU."""

import math

import pytest
import torch

import kv_reference as R
import paper_2607_23115_amd as g
from gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible GPU")
    torch.cuda.init()


def pool(gen, pages, page, heads, d, dtype, head_major):
    shape = (pages, heads, page, d) if head_major else (pages, page, heads, d)
    x = torch.randn(shape, generator=gen).to(dtype).cuda()
    return x.transpose(1, 2) if head_major else x


def check(tokens, hq, hkv, d, rot, page, dtype, interleaved=False, norm=(False, False), fused=False, head_major=True,
          seed=0, skip=False, with_q=True, in_place=False):
    say("kv_append", tokens, hq, hkv, d, rot, page, dtype, interleaved, norm, fused, head_major)
    gen = torch.Generator().manual_seed(seed)
    rows = torch.randn(tokens, hq + 2 * hkv, d, generator=gen).to(dtype).cuda()
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    pages = -(-tokens // page) + 2
    kp, vp = (pool(gen, pages, page, hkv, d, dtype, head_major) for _ in range(2))
    slots = torch.randperm(pages * page, generator=gen)[:tokens]
    if skip:
        slots[::3] = -1
        slots[1::7] = pages * page  # beyond the cache
    table = g.rotary_table(300, rot) if rot else None
    positions = torch.randint(0, 300, (tokens,), generator=gen, dtype=torch.int32)
    weight = [(1 + 0.3 * torch.randn(d, generator=gen)).to(dtype).cuda() if w else None for w in norm]
    want_k, want_v = kp.cpu().double(), vp.cpu().double()
    tol_k = torch.zeros_like(want_k)
    cpu = lambda t: None if t is None else t.cpu()  # noqa: E731
    q_want, q_tol = R.heads(q.cpu(), cpu(weight[0]), 1e-6, cpu(table), positions, interleaved)
    k_want, k_tol = R.heads(k.cpu(), cpu(weight[1]), 1e-6, cpu(table), positions, interleaved)
    for t in range(tokens):
        s = int(slots[t])
        if 0 <= s < pages * page:
            want_k[s // page, s % page], tol_k[s // page, s % page] = k_want[t], k_tol[t]
            want_v[s // page, s % page] = v[t].cpu().double()
    got = g.kv_append(k, v, kp, vp, slots.cuda(), q=q if with_q else None, q_out=q if in_place else None,
                      positions=positions.cuda() if rot else None, rotary=table, interleaved=interleaved,
                      q_weight=weight[0], k_weight=weight[1])
    torch.cuda.synchronize()
    if with_q:
        R.near(got, q_want, q_tol, "queries")
    else:
        assert got is None
    R.near(kp, want_k, tol_k, "keys")
    assert torch.equal(vp.cpu().double(), want_v)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("interleaved", [False, True])
def test_types_widths_and_layouts(dtype, d, interleaved):
    check(37, 8, 2, d, d, 16, dtype, interleaved, norm=(True, True), fused=True)
    check(5, 3, 3, d, d // 2, 32, dtype, interleaved, head_major=False)
    check(1, 7, 1, d, 16, 64, dtype, interleaved, norm=(False, True))


@pytest.mark.parametrize("tokens", [1, 2, 3, 255, 256, 257, 3001])
def test_counts_of_tokens(tokens):
    check(tokens, 4, 2, 128, 128, 64, torch.bfloat16, fused=True, seed=tokens)


def test_many_tokens_take_one_wave_each():
    check(9001, 2, 1, 64, 64, 128, torch.float16, norm=(True, False), fused=True)


def test_padding_keeps_the_cache():
    check(100, 4, 2, 128, 64, 16, torch.bfloat16, skip=True)


def test_without_queries_without_rotation_and_in_place():
    check(33, 4, 4, 128, 128, 16, torch.float16, with_q=False)
    check(33, 4, 4, 128, 0, 16, torch.float16, norm=(True, True))
    check(33, 4, 4, 128, 0, 16, torch.float16)
    check(33, 4, 4, 128, 128, 16, torch.float16, in_place=True)


def test_no_tokens():
    kp = torch.zeros(2, 16, 1, 64, dtype=torch.float16, device="cuda")
    k = torch.zeros(0, 1, 64, dtype=torch.float16, device="cuda")
    q = torch.zeros(0, 4, 64, dtype=torch.float16, device="cuda")
    got = g.kv_append(k, k, kp, kp.clone(), torch.zeros(0, dtype=torch.int64, device="cuda"), q=q)
    assert got.shape == (0, 4, 64)


def test_values_are_stored_bit_for_bit_and_bad_positions_give_nan():
    v = torch.tensor([math.inf, -math.inf, math.nan, -0.0, 6e-8, 65504.0, 0.0, 1.0] * 8, dtype=torch.float16)
    v = v.view(1, 1, 64).repeat(3, 1, 1).cuda()
    k = torch.ones_like(v)
    kp, vp = (torch.zeros(1, 16, 1, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    say("kv_append bad positions")
    positions = torch.tensor([9, 10, -1], dtype=torch.int32, device="cuda")
    got = g.kv_append(k, v, kp, vp, torch.arange(3, device="cuda"), q=k, positions=positions,
                      rotary=g.rotary_table(10, 32))
    assert torch.equal(vp[0, :3].view(torch.int16), v.view(torch.int16))
    for x in (got, kp[0, :3]):
        assert torch.isfinite(x[0]).all()
        assert torch.isnan(x[1:, :, :32]).all() and (x[1:, :, 32:] == 1).all()
    assert (kp[0, 3:] == 0).all()


def test_a_cache_beyond_32_bit_offsets():
    """The last page starts past 2^32 bytes (and elements) of the tensor."""
    pages, page, d = (1 << 32) // (4096 * 128) + 3, 4096, 128
    say("kv_append large cache", pages)
    kp = torch.empty(pages, page, 1, d, dtype=torch.bfloat16, device="cuda")
    vp = kp  # one storage will do: keys and values are the same rows
    kp[-1].zero_()
    kp[0].zero_()
    k = torch.randn(2, 1, d, device="cuda").to(torch.bfloat16)
    last = pages * page - 1
    g.kv_append(k, k, kp, vp, torch.tensor([last, last - 1], device="cuda"))
    torch.cuda.synchronize()
    assert torch.equal(kp[-1, -1], k[0]) and torch.equal(kp[-1, -2], k[1])
    assert int((kp[0] != 0).sum()) == 0 and int((kp[-1, :-2] != 0).sum()) == 0


@pytest.mark.parametrize("kw", [{}, {"factor": 4.0}, {"factor": 32.0, "original_positions": 4096, "magnitude": 1.25},
                                {"factor": 8.0, "original_positions": 512, "slow": 2.0, "fast": 16.0, "base": 5e5}])
def test_rotary_table(kw):
    say("rotary_table", kw)
    got = g.rotary_table(2000, 96, **kw).cpu().double()
    a = R.angles(2000, 96, kw.get("base", 10000.0), kw.get("factor", 1.0), kw.get("original_positions", 0),
                 kw.get("slow", 1.0), kw.get("fast", 32.0))
    want = torch.cat([a.cos(), a.sin()], 1) * kw.get("magnitude", 1.0)
    # one rounding to 32 bits, and the 64-bit angle's own error (a few units of 2^-52 of at most 2000)
    assert float((got - want).abs().max()) <= 2.0 ** -24 * kw.get("magnitude", 1.0) + 2000 * 2.0 ** -50
    assert g.rotary_table(0, 64).shape == (0, 64)


def test_rotary_table_far_out():
    """Angles of up to 2^20 radians, by the identity of the last row with float64's own cosine."""
    n = 1 << 20
    got = g.rotary_table(n, 64)[-3:].cpu().double()
    f = torch.tensor([10000.0 ** (-2 * i / 64) for i in range(32)], dtype=torch.float64)
    a = torch.arange(n - 3, n, dtype=torch.float64)[:, None] * f
    # f may differ in its last bit, which a million positions magnify to 2^20 * 2^-53
    assert float((got - torch.cat([a.cos(), a.sin()], 1)).abs().max()) <= 2.0 ** -24 + n * 2.0 ** -51


def test_a_captured_append_follows_its_inputs():
    d, dtype = 128, torch.bfloat16
    k, v = (torch.randn(6, 2, d, device="cuda").to(dtype) for _ in range(2))
    q = torch.randn(6, 4, d, device="cuda").to(dtype)
    kp, vp = (torch.zeros(4, 16, 2, d, dtype=dtype, device="cuda") for _ in range(2))
    slots = torch.arange(6, device="cuda")
    positions = torch.arange(6, dtype=torch.int32, device="cuda")
    table, q_out = g.rotary_table(100, d), torch.empty_like(q)
    call = lambda kc, vc, out: g.kv_append(k, v, kc, vc, slots, q=q, q_out=out, positions=positions,  # noqa: E731
                                           rotary=table)
    say("kv_append graph")
    call(kp, vp, q_out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(kp, vp, q_out)
    for step in range(3):
        k.copy_(torch.randn(6, 2, d, device="cuda"))
        slots.add_(7)
        positions.add_(step + 1)
        kc, vc, oc = kp.clone(), vp.clone(), torch.empty_like(q)
        call(kc, vc, oc)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(kp, kc) and torch.equal(vp, vc) and torch.equal(q_out, oc)


def test_on_another_stream():
    say("kv_append stream")
    side = torch.cuda.Stream()
    d, dtype = 64, torch.float16
    k, q = torch.randn(9, 2, d, device="cuda").to(dtype), torch.randn(9, 2, d, device="cuda").to(dtype)
    slots = torch.arange(9, device="cuda")
    positions = torch.arange(9, dtype=torch.int32, device="cuda")
    pools = [torch.zeros(1, 16, 2, d, dtype=dtype, device="cuda") for _ in range(4)]
    a = g.kv_append(k, k, pools[0], pools[1], slots, q=q, positions=positions, rotary=g.rotary_table(9, d))
    torch.cuda.synchronize()
    table = g.rotary_table(9, d, stream=side)
    b = g.kv_append(k, k, pools[2], pools[3], slots, q=q, positions=positions, rotary=table, stream=side)
    side.synchronize()
    assert torch.equal(a, b) and torch.equal(pools[0], pools[2]) and torch.equal(pools[1], pools[3])


def refused(message, **kw):
    d = 64
    a = {"k": torch.zeros(4, 2, d), "v": torch.zeros(4, 2, d), "k_pages": torch.zeros(3, 16, 2, d),
         "v_pages": torch.zeros(3, 16, 2, d)}
    a = {n: t.to(torch.float16).cuda() for n, t in a.items()}
    a["slots"] = torch.arange(4, device="cuda")
    a.update({n: x(a) if callable(x) else x for n, x in kw.items()})
    before = a["k_pages"].clone()
    with pytest.raises((ValueError, g.GleamError), match=message):
        g.kv_append(**a)
    torch.cuda.synchronize()
    assert torch.equal(a["k_pages"], before)


def test_refusals():
    f = torch.float16
    refused("k must be", k=lambda a: a["k"].float())
    refused("k must be", k=lambda a: a["k"][:, :1])
    refused("on the GPU", k=lambda a: a["k"].cpu())
    refused("differ in tokens", v=lambda a: a["v"][:3])
    refused("last dimension", k=lambda a: a["k"].transpose(1, 2).contiguous().transpose(1, 2))
    refused("slots holds 3", slots=lambda a: a["slots"][:3])
    refused("slots must be", slots=lambda a: a["slots"].int())
    refused("page_tokens", k_pages=lambda a: a["k_pages"][:, :8], v_pages=lambda a: a["v_pages"][:, :8])
    refused("differ in shape", v_pages=lambda a: a["v_pages"][:2])
    refused("overlap", k_pages=lambda a: a["k_pages"][:, :, :1].expand(-1, -1, 2, -1))
    refused("need q", q_weight=lambda a: torch.ones(64, dtype=f, device="cuda"))
    refused("k_weight holds", k_weight=lambda a: torch.ones(32, dtype=f, device="cuda"))
    refused("positions is required", rotary=lambda a: g.rotary_table(8, 64))
    refused("rot_dim", rotary=lambda a: g.rotary_table(8, 24), positions=lambda a: a["slots"].int())
    refused("rot_dim", rotary=lambda a: g.rotary_table(8, 128), positions=lambda a: a["slots"].int())
    refused("aligned", k=lambda a: torch.zeros(4 * 128 + 1, dtype=f, device="cuda")[1:].view(4, 2, 64))
    refused("multiples of 8", k=lambda a: torch.zeros(4, 2, 68, dtype=f, device="cuda")[:, :, :64])
    refused("q_out and q", q=lambda a: a["k"], q_out=lambda a: a["k"][:3])
    for bad in ({"rot_dim": 3}, {"rot_dim": 64, "base": 0.0}, {"rot_dim": 64, "factor": -1.0},
                {"rot_dim": 64, "factor": math.nan}, {"rot_dim": 64, "slow": 2.0, "fast": 2.0}):
        with pytest.raises(g.GleamError):
            g.rotary_table(8, **bad)


def test_gradients_are_refused_and_not_dropped():
    f = torch.float16
    a = {"k": torch.zeros(4, 2, 64), "v": torch.zeros(4, 2, 64), "q": torch.zeros(4, 2, 64),
         "k_pages": torch.zeros(3, 16, 2, 64), "v_pages": torch.zeros(3, 16, 2, 64), "q_weight": torch.ones(64),
         "k_weight": torch.ones(64)}
    a = {n: t.to(f).cuda() for n, t in a.items()}
    a.update(slots=torch.arange(4, device="cuda"), positions=torch.arange(4, dtype=torch.int32, device="cuda"),
             rotary=g.rotary_table(4, 64))
    say("kv_append gradients")
    for name in ("k", "v", "q", "k_pages", "v_pages", "q_weight", "k_weight", "rotary"):
        b = {**a, name: a[name].clone().requires_grad_()}
        with pytest.raises(ValueError, match=name + " requires a gradient"):
            g.kv_append(**b)
        with torch.no_grad():
            assert not g.kv_append(**b).requires_grad
        with torch.autograd.forward_ad.dual_level():
            b[name] = torch.autograd.forward_ad.make_dual(a[name], torch.ones_like(a[name]))
            with pytest.raises(ValueError, match=name + " requires a gradient"):
                g.kv_append(**b)
    refused("q_out requires a gradient", q=lambda a: a["k"], q_out=lambda a: a["k"].clone().requires_grad_())
    with torch.inference_mode():
        g.kv_append(**a)


def test_a_table_without_positions_gives_nan():
    say("kv_append empty table")
    k = torch.ones(3, 2, 64, dtype=torch.float16, device="cuda")
    kp, vp = (torch.zeros(1, 16, 2, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    positions = torch.tensor([0, 5, -1], dtype=torch.int32, device="cuda")
    got = g.kv_append(k, k, kp, vp, torch.arange(3, device="cuda"), q=k, positions=positions,
                      rotary=g.rotary_table(0, 32))
    for x in (got, kp[0, :3]):
        assert torch.isnan(x[..., :32]).all() and (x[..., 32:] == 1).all()
    refused("rot_dim", rotary=lambda a: g.rotary_table(0, 24), positions=lambda a: a["slots"].int())
    refused("rot_dim", rotary=lambda a: torch.empty(0, 0, device="cuda"), positions=lambda a: a["slots"].int())


def test_a_cache_without_pages():
    say("kv_append without pages")
    none = torch.empty(0, 16, 2, 64, dtype=torch.float16, device="cuda")
    k = torch.randn(3, 2, 64, device="cuda").to(torch.float16)
    got = g.kv_append(k, k, none, none, torch.tensor([0, 5, -1], device="cuda"), q=k)
    torch.cuda.synchronize()
    assert torch.equal(got, k)
