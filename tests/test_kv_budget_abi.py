"""The calls on trees of drafts and on the cache's budget, on the CPU: arguments are checked before anything
is enqueued, and the binding's structures are laid out as the header's. The plain computations that the GPU
tests compare with are held against small cases written out."""

import ctypes
import inspect
import math
import os
import shutil
import subprocess

import pytest
import torch

import budget_reference as B
import paper_2607_23115_amd as g
from test_kv_abi import BAD_CACHES, attend, batch, kv, put

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def tree(parent=256, q_first=256, n_tokens=4, n_seq=2, seen=256, words=1, depth=256):
    return g.lib.gleam_draft_tree(parent, q_first, n_tokens, n_seq, seen, words, depth, None)


def tree_attend(cache=None, seen=256, words=1, out=256, ws=256, ws_bytes=1 << 40, **kw):
    return g.lib.gleam_tree_attention(ctypes.byref(cache if cache is not None else kv()), ctypes.byref(batch(**kw)), seen,
                                      words, out, None, ws, ws_bytes, None)


def accept(cache=None, **kw):
    a = put(g._Accept(256, 256, 256, 256, 256, 512, 4, 2, 3, 1), **kw)
    return g.lib.gleam_kv_accept(ctypes.byref(cache if cache is not None else kv()), ctypes.byref(a), None)


def weigh(cache=None, **kw):
    a = put(g._Weigh(256, 256, 256, 256, 256, 1 << 20, 1 << 20, 256, 256, 4, 2, 3, 128, 64, 4, 1.0), **kw)
    return g.lib.gleam_kv_weigh(ctypes.byref(cache if cache is not None else kv()), ctypes.byref(a), None)


def evict_args(**kw):
    return put(g._Evict(256, 256, 1 << 20, 1 << 21, 256, 1 << 20, 1 << 21, 512, 2, 3, 20, 0, 0), **kw)


def evict(cache=None, ws=256, ws_bytes=1 << 40, **kw):
    return g.lib.gleam_kv_evict(ctypes.byref(cache if cache is not None else kv()), ctypes.byref(evict_args(**kw)), ws,
                                ws_bytes, None)


def evict_ws(cache=None, **kw):
    return g.lib.gleam_kv_evict_ws_bytes(ctypes.byref(cache if cache is not None else kv()),
                                         ctypes.byref(evict_args(**kw)))


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_caches_that_are_refused(bad):
    for call in (tree_attend, accept, weigh, evict):
        assert call(kv(**bad)) == g.E_INVALID
    assert evict_ws(kv(**bad)) == 0


def test_trees_that_are_refused():
    for bad in ({"parent": None}, {"q_first": None}, {"seen": None}, {"seen": 260}, {"words": 0}):
        assert tree(**bad) == g.E_INVALID
        assert b"gleam_draft_tree" in g.lib.gleam_last_error()
    assert tree(n_seq=(1 << 20) + 1) == g.E_UNSUPPORTED
    assert tree(n_tokens=1 << 31) == g.E_UNSUPPORTED
    assert tree(words=65537) == g.E_UNSUPPORTED
    assert tree(n_tokens=0, seen=None) == g.OK


@pytest.mark.parametrize("bad", [{"seen": None}, {"seen": 260}, {"words": 0}, {"q": None}, {"q": 8}, {"q_stride": (4, 64)},
                                 {"q_heads": 3}, {"q_first": None}, {"own_len": None}, {"own_pages": None},
                                 {"group_first": None}, {"prefix_len": None}, {"own_width": 1 << 27}, {"out": 8},
                                 {"ws": 300}])
def test_tree_attention_that_is_refused(bad):
    assert tree_attend(**bad) == g.E_INVALID
    assert b"gleam_tree_attention" in g.lib.gleam_last_error()


def test_tree_attention_limits():
    assert tree_attend(words=65537) == g.E_UNSUPPORTED
    assert tree_attend(n_tokens=1 << 30) == g.E_UNSUPPORTED
    need = [g.lib.gleam_tree_attention_ws_bytes(ctypes.byref(kv()), ctypes.byref(batch(n_tokens=t))) for t in (4, 400)]
    assert need[0] == g.lib.gleam_prefix_attention_ws_bytes(ctypes.byref(kv()), ctypes.byref(batch()))
    assert need[1] > g.lib.gleam_prefix_attention_ws_bytes(ctypes.byref(kv()), ctypes.byref(batch(n_tokens=400)))
    for t, n in zip((4, 400), need):
        assert tree_attend(n_tokens=t, ws_bytes=n - 1) == g.E_WORKSPACE
    assert g.lib.gleam_tree_attention_ws_bytes(ctypes.byref(kv(head_dim=96)), ctypes.byref(batch())) == 0
    assert tree_attend(n_tokens=0, seen=None) == g.OK
    assert attend(n_tokens=0) == g.OK


@pytest.mark.parametrize("bad", [{"q_first": None}, {"seen": None}, {"seen": 257}, {"seen_words": 0}, {"leaf": None},
                                 {"own_pages": None}, {"own_len": None}, {"len_out": None}, {"len_out": 256},
                                 {"len_out": 260}, {"own_width": 1 << 27}])
def test_accepted_paths_that_are_refused(bad):
    assert accept(**bad) == g.E_INVALID
    assert b"gleam_kv_accept" in g.lib.gleam_last_error()


@pytest.mark.parametrize("name", ["own_len", "leaf", "q_first", "seen", "own_pages"])
def test_an_accepted_length_written_over_what_is_read(name):
    """len_out of 2 sequences is 8 bytes; the fields: 2, 2 and 3 of 4 bytes, 4 of 8, 6 of 4."""
    size = {"own_len": 8, "leaf": 8, "q_first": 12, "seen": 32, "own_pages": 24}[name]
    for to in (1 << 20, (1 << 20) - 4, (1 << 20) + size - 4):
        assert accept(**{name: 1 << 20, "len_out": to}) == g.E_INVALID
        assert name.encode() in g.lib.gleam_last_error() and b"overlap" in g.lib.gleam_last_error()


def test_accept_limits():
    assert accept(kv(k_stride=(2048, 64, 64))) == g.E_INVALID
    assert b"overlap" in g.lib.gleam_last_error()
    assert accept(n_seq=(1 << 20) + 1) == g.E_UNSUPPORTED
    assert accept(n_tokens=1 << 31) == g.E_UNSUPPORTED
    assert accept(n_seq=0) == g.OK


@pytest.mark.parametrize("bad", [{"q": None}, {"q": 8}, {"q_stride": (-8, 64)}, {"q_heads": 3}, {"q_heads": 0},
                                 {"q_heads": 1 << 16}, {"q_first": None}, {"own_len": None}, {"own_pages": None},
                                 {"lse": None}, {"weights": None}, {"weights_out": None}, {"weights": (1 << 20) + 2},
                                 {"weights_out": (1 << 20) + 4}, {"weights_out": (1 << 20) - 4}, {"born": None},
                                 {"positions": None}, {"born": 258}, {"own_width": 1 << 27}])
def test_weights_that_are_refused(bad):
    assert weigh(**bad) == g.E_INVALID
    assert b"gleam_kv_weigh" in g.lib.gleam_last_error()


def test_weigh_limits():
    assert weigh(n_tokens=1 << 30) == g.E_UNSUPPORTED
    assert weigh(n_seq=(1 << 20) + 1) == g.E_UNSUPPORTED
    assert weigh(kv(k_stride=(1 << 40, 1 << 26, 64))) == g.E_UNSUPPORTED
    for nothing in ({"n_seq": 0}, {"own_width": 0}):
        assert weigh(**nothing) == g.OK
    assert weigh(kv(n_pages=0)) == g.OK


@pytest.mark.parametrize("bad", [{"own_len": None}, {"own_pages": None}, {"weights": None}, {"born": None},
                                 {"total": None}, {"weights_out": None}, {"born_out": None}, {"len_out": None},
                                 {"len_out": 256}, {"len_out": 260},
                                 {"weights_out": (1 << 20) + 4}, {"born_out": (1 << 21) - 4}, {"weights": (1 << 20) + 1},
                                 {"own_width": 1 << 27}, {"ws": None}, {"ws": 128}])
def test_evictions_that_are_refused(bad):
    assert evict(**bad) == g.E_INVALID
    assert b"gleam_kv_evict" in g.lib.gleam_last_error()


@pytest.mark.parametrize("name", ["own_len", "total", "own_pages"])
def test_a_budgets_length_written_over_what_is_read(name):
    size = {"own_len": 8, "total": 8, "own_pages": 24}[name]
    for to in (1 << 22, (1 << 22) - 4, (1 << 22) + size - 4):
        assert evict(**{name: 1 << 22, "len_out": to}) == g.E_INVALID
        assert name.encode() in g.lib.gleam_last_error() and b"overlap" in g.lib.gleam_last_error()


def test_what_is_empty_does_not_overlap():
    """A table without pages at the lengths' address: the call goes on to the next thing that it checks."""
    assert evict(own_width=0, own_pages=512, ws=None) == g.E_INVALID
    assert b"workspace" in g.lib.gleam_last_error()


def test_eviction_workspaces_and_limits():
    assert evict(kv(v_stride=(2048, 128, 0))) == g.E_INVALID
    assert b"overlap" in g.lib.gleam_last_error()
    need = evict_ws()
    assert need % 256 == 0 and need >= 2 * 2 * 20 * 8
    assert evict(ws_bytes=need - 1) == g.E_WORKSPACE
    assert evict(n_seq=(1 << 20) + 1) == g.E_UNSUPPORTED
    big = kv(kv_heads=4096, k_stride=(16 * 4096 * 64, 4096 * 64, 64), v_stride=(16 * 4096 * 64, 4096 * 64, 64))
    assert evict(big, n_seq=1 << 20) == g.E_UNSUPPORTED
    assert evict(n_seq=1 << 20, own_width=1 << 20, keep=1 << 23) == g.E_UNSUPPORTED
    assert evict_ws(n_seq=1 << 20, own_width=1 << 20, keep=1 << 23) == 0
    assert evict(n_seq=0) == g.OK
    # no more than may move: none where the tables hold no more than is kept
    assert evict_ws(keep=48) == evict_ws(keep=0) == 256
    assert evict_ws(own_width=100, keep=1000) < evict_ws(own_width=200, keep=1000)


def test_structures_match_the_header(tmp_path):
    cc = shutil.which("gcc")
    assert cc, "gcc not found"
    fields = {"gleam_accept": (g._Accept, ["d_len_out len_out", "n_tokens", "own_width", "seen_words"]),
              "gleam_weigh": (g._Weigh, ["d_lse lse", "d_positions positions", "n_tokens", "q_stride q_token", "q_heads",
                                         "scale"]),
              "gleam_evict": (g._Evict, ["d_total total", "d_born_out born_out", "d_len_out len_out", "n_seq", "keep",
                                         "recent"])}
    lines = [f'printf("%zu\\n", sizeof({s}));' for s in fields]
    lines += [f'printf("%zu\\n", offsetof({s}, {f.split()[0]}));' for s, (_, fs) in fields.items() for f in fs]
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "gleam.h"\nint main(void) {' + "".join(lines) +
                   "return 0;}\n")
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True).stdout.split()]
    want = [ctypes.sizeof(t) for t, _ in fields.values()]
    want += [getattr(t, f.split()[-1]).offset for t, fs in fields.values() for f in fs]
    assert got == want


def test_the_binding_refuses_host_tensors():
    x = torch.zeros(2, 16, 1, 64, dtype=torch.float16)
    i, f = torch.zeros(4, dtype=torch.int32), torch.zeros(2, 1, 16)
    seen = torch.zeros(4, 1, dtype=torch.int64)
    for call in (lambda: g.draft_tree(i, i, 4), lambda: g.tree_attention(x[0, :4], x, x, i, seen, i, i),
                 lambda: g.kv_accept(x, x, i, seen, i, i, i), lambda: g.kv_weigh(x[0, :4], x, i, i, i, f, f),
                 lambda: g.kv_evict(x, x, i, i, f, i, i, 3)):
        with pytest.raises(ValueError, match="on the GPU"):
            call()


def i32(x):
    return torch.tensor(x, dtype=torch.int32)


def test_public_calls_have_no_private_parameters():
    for call in (g.prefix_attention, g.tree_attention, g.draft_tree, g.kv_accept, g.kv_weigh, g.kv_evict, g.kv_append):
        assert not [p for p in inspect.signature(call).parameters if p.startswith("_")], call.__name__


def test_a_small_tree_written_out():
    seen, depth = B.tree(i32([-1, 0, 0, 1, 9, -1, 0]), i32([0, 5, 7]), 2)
    assert seen[:, 0].tolist() == [0b1, 0b11, 0b101, 0b1011, 0b10000, 0b1, 0b11] and (seen[:, 1] == 0).all()
    assert depth.tolist() == [0, 1, 1, 2, 0, 0, 1]
    seen, _ = B.tree(torch.arange(-1, 63, dtype=torch.int32), i32([0, 64]), 1)
    assert seen[63].item() == -1 and seen[62].item() == (1 << 63) - 1


def test_small_sums_and_evictions_written_out():
    k = torch.zeros(1, 16, 1, 64, dtype=torch.float16)
    k[0, :3, 0, 0] = torch.tensor([1.0, 2.0, 3.0])
    q = torch.zeros(2, 1, 64, dtype=torch.float16)
    q[:, 0, 0] = torch.tensor([1.0, 2.0])
    w, b = torch.full((1, 1, 16), 5.0), torch.full((1, 1, 16), -1, dtype=torch.int32)
    out, born, tol = B.weigh(q, k, i32([0, 2]), i32([[0]]), i32([3]), torch.tensor([[0.5], [math.inf]]), w, b, i32([8, 9]),
                             scale=1.0)
    assert out[0, 0, :4].tolist() == pytest.approx([5 + math.exp(0.5), math.exp(1.5), 0.0, 5.0])
    assert born[0, 0, :4].tolist() == [-1, 8, 9, -1] and tol[0, 0, 3] == 0
    w = torch.tensor([[[3.0, 1.0, 1.0, math.nan, 2.0, 1.0] + [0.0] * 10]])
    b = torch.arange(16, dtype=torch.int32).view(1, 1, 16)
    v = torch.arange(16.0, dtype=torch.float16).view(1, 16, 1, 1).expand(1, 16, 1, 64).contiguous()
    kp, vp, ww, bb, n = B.evict(v, v, i32([[0]]), i32([6]), w, b, i32([6]), 3)
    assert n.tolist() == [3] and vp[0, :3, 0, 0].tolist() == [0, 1, 4] and bb[0, 0, :3].tolist() == [0, 1, 4]
    kp, vp, ww, bb, n = B.evict(v, v, i32([[0]]), i32([6]), w, b, i32([6]), 3, 2, 1)
    assert vp[0, :3, 0, 0].tolist() == [0, 1, 5] and ww[0, 0, :3].tolist() == [3, 1, 1]
    seen = torch.tensor([[0b1], [0b11], [0b101], [0b1101]])
    kp, vp, n = B.accept(v, v, i32([0, 4]), seen, i32([3]), i32([[0]]), i32([10]))
    assert n.tolist() == [9] and vp[0, 5:11, 0, 0].tolist() == [5, 6, 8, 9, 9, 10]
