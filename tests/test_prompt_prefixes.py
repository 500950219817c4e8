"""Blocks of prompts identified together with all that comes before them (Batch.prefixes): a
block's own digest is the same behind any other, while its cached keys and values are not."""

import numpy as np
import pytest
import torch

import oracle
import paper_2607_23115_amd as g
from gpu_util import keys_to_device, say, to_device, u64

BLOCK, TOKENS = 4096, 1024


def prompt(rng, *parts):
    """Blocks by name ("A" is the same tokens everywhere), numbers are so many tokens of their own."""
    return np.concatenate([np.random.default_rng(ord(x)).integers(0, 32000, TOKENS, dtype=np.int32)
                           if isinstance(x, str) else rng.integers(0, 32000, x, dtype=np.int32) for x in parts])


def lists(prompts):
    """Every block's own digest and list of digests, as the oracle has them."""
    payloads = [p.view(np.uint8) for p in prompts]
    digests = oracle.batch_digests(payloads, BLOCK)[0]
    first = oracle.geometry([p.size for p in payloads], BLOCK)[0]
    at, lens = g._digest_lists(first)
    raw = digests.view(np.uint8)
    return digests, [raw[int(a):int(a) + int(n)] for a, n in zip(at, lens)]


def test_a_blocks_own_digest_is_the_same_behind_any_other():
    rng = np.random.default_rng(1)
    digests, of = lists([prompt(rng, "A", "B"), prompt(rng, "C", "B"), prompt(rng, "A", "B", 30), prompt(rng, "B")])
    assert digests[1] == digests[3] == digests[5] == digests[7]
    ids = [oracle.xxh64(x) for x in of]
    assert len({ids[1], ids[3], ids[7]}) == 3  # B behind A, behind C and at the start
    assert ids[0] == ids[4] and ids[1] == ids[5] and ids[6] not in ids[:6]


def test_lists_of_digests():
    at, lens = g._digest_lists(np.array([0, 3, 3, 4, 6], np.uint64))
    assert at.tolist() == [0, 0, 0, 24, 32, 32] and lens.tolist() == [8, 16, 24, 8, 8, 16]
    at, lens = g._digest_lists(np.array([0], np.uint64))
    assert at.size == 0 and lens.size == 0


def batch_of(prompts):
    lens = np.array([4 * p.size for p in prompts])
    offs = np.concatenate([[0], np.cumsum(lens)[:-1]])
    return g.Batch.from_arena(to_device(np.concatenate(prompts).view(np.uint8)), offs, lens, BLOCK)


@pytest.mark.gpu
def test_held_blocks_are_found_behind_what_they_were_computed_behind():
    """The table holds A|B and C|D: of a prompt A|D only the first block's pages may be used."""
    say("prompt prefixes")
    rng = np.random.default_rng(2)
    held = batch_of([prompt(rng, "A", "B"), prompt(rng, "C", "D")])
    table = g.Cache(1 << 8)
    table.insert(g.fp_chunks(g.Batch.prefixes(held, g.fp_chunks(held))), keys_to_device(np.arange(0, 64, 16)))
    asked = [prompt(rng, "A", "D"), prompt(rng, "C", "D", 7), prompt(rng, "A", "B", "D"), prompt(rng, "D"),
             prompt(rng, "A")[:1000]]
    batch = batch_of(asked)
    own = g.fp_chunks(batch)
    found = g.detect(g.Batch.prefixes(batch, own), table)
    torch.cuda.synchronize()
    digests, of = lists(asked)
    assert np.array_equal(u64(own), digests)
    assert np.array_equal(u64(found.digests)[:batch.n_blocks], [oracle.xxh64(x) for x in of])
    status, ref = found.status[:batch.n_blocks].cpu().numpy(), u64(found.ref)
    assert (status == g.HIT_CACHE).tolist() == [True, False, True, True, False, True, True, False, False, False]
    assert ref[[0, 2, 3, 5, 6]].tolist() == [0, 32, 48, 0, 16]


@pytest.mark.gpu
def test_long_prompts_and_empty_ones():
    """Lists of more digests than a leaf, and than a block of the prompts, holds."""
    say("prompt prefixes, long")
    rng = np.random.default_rng(3)
    prompts = [prompt(rng, 1100 * TOKENS + 5), prompt(rng, 3)[:0], prompt(rng, 2 * TOKENS)]
    batch = batch_of(prompts)
    ids = g.Batch.prefixes(batch, g.fp_chunks(batch))
    assert ids.n_blocks == batch.n_blocks == 1103 and ids.block_bytes == 16384
    got = u64(g.fp_chunks(ids))
    want = oracle.batch_digests([x.copy() for x in lists(prompts)[1]], 16384)[0]
    assert np.array_equal(got, want)
    none = batch_of([prompt(rng, 3)[:0]])
    assert g.Batch.prefixes(none, g.fp_chunks(none)).n_blocks == 0
    with pytest.raises(ValueError, match="digests holds"):
        g.Batch.prefixes(batch, g.fp_chunks(batch)[:-1])
    with pytest.raises(ValueError, match="on the GPU"):
        g.Batch.prefixes(batch, torch.zeros(batch.n_blocks, dtype=torch.int64))
