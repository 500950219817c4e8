"""The paged key/value cache's calls on the CPU: arguments are checked before anything is
enqueued, and the binding's structures are laid out as the header's."""

import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2607_23115_amd as g

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def put(s, **kw):
    """Sets fields; "k_stride" and its like are all strides of k, in their order."""
    for n, x in kw.items():
        if n.endswith("_stride"):
            names = [f for f, _ in s._fields_ if f in (n[0] + "_page", n[0] + "_place", n[0] + "_token", n[0] + "_head")]
            assert len(names) == len(x)
            put(s, **dict(zip(names, x)))
        else:
            setattr(s, n, x)
    return s


def kv(**kw):
    return put(g._KvPages(256, 256, 4, 16, 2, 64, 0, 2048, 128, 64, 2048, 128, 64), **kw)


def append(cache=None, **kw):
    a = put(g._Append(256, 256, 256, 256, 256, 256, 256, None, None, 4, 10, 128, 64, 128, 64, 128, 64, 2, 64, 0, 1e-6),
            **kw)
    return g.lib.gleam_kv_append(ctypes.byref(cache if cache is not None else kv()), ctypes.byref(a), None)


def batch(**kw):
    return put(g._PrefixBatch(256, 256, 256, 256, 256, 256, 256, 4, 2, 1, 3, 3, 128, 64, 4, 1.0), **kw)


def attend(cache=None, out=256, ws=256, ws_bytes=1 << 40, **kw):
    return g.lib.gleam_prefix_attention(ctypes.byref(cache if cache is not None else kv()), ctypes.byref(batch(**kw)), out,
                                        None, ws, ws_bytes, None)


BAD_CACHES = [{"dtype": 2}, {"head_dim": 96}, {"head_dim": 0}, {"kv_heads": 0}, {"kv_heads": 1 << 16},
              {"page_tokens": 8}, {"page_tokens": 24}, {"page_tokens": 8192}, {"k": None}, {"v": 8},
              {"n_pages": 1 << 31}, {"k_stride": (2048, 4, 64)}, {"v_stride": (-2048, 128, 64)}]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_caches_that_are_refused(bad):
    assert append(kv(**bad)) == g.E_INVALID
    assert attend(kv(**bad)) == g.E_INVALID
    assert b"gleam_prefix_attention" in g.lib.gleam_last_error()
    assert g.lib.gleam_prefix_attention_ws_bytes(ctypes.byref(kv(**bad)), ctypes.byref(batch())) == 0


@pytest.mark.parametrize("bad", [{"k": None}, {"v": 264}, {"slots": None}, {"q_out": None}, {"q": None},
                                 {"q_heads": 0}, {"positions": None}, {"rot_dim": 0}, {"rot_dim": 72}, {"rot_dim": 80},
                                 {"rotary": 260}, {"k_stride": (128, 60)}, {"q_stride": (-8, 64)}, {"q_weight": 258},
                                 {"q_heads": 1 << 16}])
def test_appends_that_are_refused(bad):
    assert append(**bad) == g.E_INVALID
    assert b"gleam_kv_append" in g.lib.gleam_last_error()


def test_appends_into_overlapping_places_are_refused():
    assert append(kv(k_stride=(2048, 128, 0))) == g.E_INVALID
    assert append(kv(v_stride=(0, 128, 64))) == g.E_INVALID
    assert append(kv(v_stride=(2048, 0, 64))) == g.E_INVALID
    assert append(n_tokens=1 << 31) == g.E_UNSUPPORTED
    assert append(n_tokens=0) == g.OK


@pytest.mark.parametrize("bad", [{"q": None}, {"q": 8}, {"q_stride": (4, 64)}, {"q_heads": 3}, {"q_heads": 0},
                                 {"q_first": None}, {"own_len": None}, {"own_pages": None}, {"group_first": None},
                                 {"prefix_len": None}, {"prefix_pages": None}, {"own_width": 1 << 27},
                                 {"prefix_width": 1 << 27}])
def test_attention_that_is_refused(bad):
    assert attend(**bad) == g.E_INVALID
    assert b"gleam_prefix_attention" in g.lib.gleam_last_error()


def test_attention_workspaces_and_limits():
    assert attend(out=None) == g.E_INVALID
    assert attend(out=8) == g.E_INVALID
    assert attend(ws=None) == g.E_INVALID
    assert attend(ws=300) == g.E_INVALID
    need = g.lib.gleam_prefix_attention_ws_bytes(ctypes.byref(kv()), ctypes.byref(batch()))
    assert need > 0 and need % 256 == 0
    assert attend(ws_bytes=need - 1) == g.E_WORKSPACE
    assert attend(n_tokens=1 << 30) == g.E_UNSUPPORTED
    assert attend(n_seq=(1 << 20) + 1) == g.E_UNSUPPORTED
    assert attend(n_groups=(1 << 20) + 1) == g.E_UNSUPPORTED
    assert attend(n_tokens=0) == g.OK
    sizes = [g.lib.gleam_prefix_attention_ws_bytes(ctypes.byref(kv()), ctypes.byref(batch(n_tokens=t, n_seq=t)))
             for t in (1, 10, 1000, 100_000)]
    assert sizes == sorted(sizes)


def test_rotary_tables_that_are_refused():
    f = g.lib.gleam_rotary_table
    assert f(None, 4, 64, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0, None) == g.E_INVALID
    assert f(256, 4, 63, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0, None) == g.E_INVALID
    assert f(256, 1 << 31, 64, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0, None) == g.E_INVALID
    assert f(256, 4, 64, 1e4, 0.0, 0.0, 1.0, 32.0, 1.0, None) == g.E_INVALID
    assert f(256, 4, 64, 1e4, 1.0, float("nan"), 1.0, 32.0, 1.0, None) == g.E_INVALID
    assert f(256, 4, 64, 1e4, 1.0, 0.0, 32.0, 32.0, 1.0, None) == g.E_INVALID
    assert f(None, 0, 64, 1e4, 1.0, 0.0, 1.0, 32.0, 1.0, None) == g.OK


def test_structures_match_the_header(tmp_path):
    cc = shutil.which("gcc")
    assert cc, "gcc not found"
    fields = {"gleam_kv_pages": (g._KvPages, ["n_pages", "page_tokens", "dtype", "k_stride k_page",
                                              "v_stride v_page"]),
              "gleam_append": (g._Append, ["n_tokens", "rotary_positions", "q_stride q_token", "v_stride v_token",
                                           "q_heads", "eps"]),
              "gleam_prefix_batch": (g._PrefixBatch, ["n_tokens", "prefix_width", "q_stride q_token", "q_heads",
                                                      "scale"])}
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
    with pytest.raises(ValueError, match="on the GPU"):
        g.kv_append(x[0, :4], x[0, :4], x, x, torch.zeros(4, dtype=torch.int64))
    with pytest.raises(ValueError, match="on the GPU"):
        g.prefix_attention(x[0, :4], x, x, None, None, None)
    with pytest.raises(ValueError, match="CUDA device"):
        g.rotary_table(4, 64, device="cpu")


def test_appends_into_places_that_overlap_by_their_strides_together_are_refused():
    # each stride holds a head by itself
    for bad in ((2048, 64, 64),       # head 1 of a place is head 0 of the next
                (2048, 64, 512),      # head 1 starts within head 0's places
                (1024, 128, 64),      # a page's second half is the next page
                (64, 128, 64), (1984, 128, 64), (128, 256, 64)):
        assert append(kv(k_stride=bad)) == g.E_INVALID, bad
        assert append(kv(v_stride=bad)) == g.E_INVALID, bad
        assert b"overlap" in g.lib.gleam_last_error()


@pytest.mark.parametrize("good", [(2048, 128, 64), (2048, 64, 1024), (4096, 256, 64), (64, 512, 256), (128, 512, 64),
                                  (1 << 40, 1 << 20, 64), ((1 << 62) - 8, 128, 64)])
def test_orders_of_pages_places_and_heads_that_do_not_overlap_are_taken(good):
    # what the next check refuses, so that nothing is launched
    assert append(kv(k_stride=good, v_stride=good), n_tokens=1 << 31) == g.E_UNSUPPORTED
    # strides of dimensions of one multiply nothing
    one = put(kv(k_stride=(0, 64, 0), v_stride=(8, 64, 8)), n_pages=1, kv_heads=1)
    assert append(one, n_tokens=1 << 31) == g.E_UNSUPPORTED


def test_small_batches_ask_for_small_workspaces():
    """A unit leaves no more rows of partial results than the batch has, of 256 units twice over."""
    for d in (64, 128, 256):
        cache = kv(head_dim=d, kv_heads=8, k_stride=(16 * 8 * d, d, 16 * d), v_stride=(16 * 8 * d, d, 16 * d))
        for tokens, q_heads in ((1, 8), (1, 32), (3, 16)):
            need = g.lib.gleam_prefix_attention_ws_bytes(ctypes.byref(cache), ctypes.byref(
                batch(n_tokens=tokens, n_seq=1, n_groups=0, q_heads=q_heads, own_width=1 << 14)))
            assert 0 < need <= 2 * 256 * (tokens * q_heads // 8) * (4 * d + 8) + 4096
