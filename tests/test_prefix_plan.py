"""The arithmetic by which prefix_attention cuts its work, compiled by itself for the CPU: over
random batches, units and partial results stay within what the launch and the workspace are
sized for, and the chunks of an item cover its steps."""

import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_23115_amd", "csrc")

# reads: head_dim kv_heads ratio target n_seq n_groups, then per sequence tokens own, then per group
# sequences prefix (groups cover the first sequences in order)
BODY = r"""
#include <cstdio>
#include <vector>
#include "prefix_plan.h"
using namespace gleam;
struct It { uint64_t tokens, prefix, own; bool partial; };
int main() {
  unsigned long long dim, kvh, ratio, target, ns, ng;
  if (scanf("%llu %llu %llu %llu %llu %llu", &dim, &kvh, &ratio, &target, &ns, &ng) != 6) return 2;
  std::vector<It> items(ng + ns);
  uint64_t all = 0;
  for (uint64_t s = 0; s < ns; ++s) {
    unsigned long long t, o;
    if (scanf("%llu %llu", &t, &o) != 2) return 2;
    items[ng + s] = {t, 0, o, false};
    all += t;
  }
  uint64_t at = 0;
  for (uint64_t g = 0; g < ng; ++g) {
    unsigned long long n, p;
    if (scanf("%llu %llu", &n, &p) != 2) return 2;
    uint64_t tokens = 0;
    for (uint64_t s = at; s < at + n; ++s) tokens += items[ng + s].tokens;
    const bool joint = joint_group(tokens * ratio, n);
    items[g] = {tokens, joint ? 0 : p, 0, true};
    for (uint64_t s = at; s < at + n; ++s) {
      if (joint) items[ng + s].prefix = p;
      else items[ng + s].partial = p > 0;
    }
    at += n;
  }
  uint64_t cost[2] = {0, 0};
  for (const It& it : items)
    if (it.tokens) cost[few_rows((uint32_t)(it.tokens * ratio))] += item_cost((uint32_t)(it.tokens * ratio), steps_of((uint32_t)it.prefix) + steps_of((uint32_t)it.own)) * kvh;
  uint64_t units = 0, parts = 0;
  for (const It& it : items) {
    const uint32_t rows = (uint32_t)(it.tokens * ratio);
    const uint32_t steps = it.tokens ? steps_of((uint32_t)it.prefix) + steps_of((uint32_t)it.own) : 0;
    const Cut c = cut_steps(steps, chunk_steps(rows, cost[few_rows(rows)], (uint32_t)target, (uint32_t)dim));
    if ((steps == 0) != (c.chunks == 0)) return 3;
    if (steps && ((uint64_t)c.chunks * c.per < steps || (uint64_t)(c.chunks - 1) * c.per >= steps)) return 4;
    units += (uint64_t)tiles_of(rows) * kvh * c.chunks;
    if (it.partial || c.chunks > 1) parts += rows * kvh * c.chunks;
  }
  uint64_t longest[2] = {0, 0};
  for (const It& it : items) {
    if (steps_of((uint32_t)it.own) > longest[0]) longest[0] = steps_of((uint32_t)it.own);
    if (steps_of((uint32_t)it.prefix) > longest[1]) longest[1] = steps_of((uint32_t)it.prefix);
  }
  PlanShape s{all, ns, ng, (uint32_t)kvh, (uint32_t)ratio, (uint32_t)target, (uint32_t)(longest[0] + longest[1]), (uint32_t)dim};
  printf("%llu %llu %llu %llu\n", (unsigned long long)units, (unsigned long long)most_units(s),
         (unsigned long long)parts, (unsigned long long)most_partials(s));
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++")
    assert cxx, "g++ not found"
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(BODY)
    subprocess.run([cxx, "-std=c++17", "-Wall", "-Werror", "-O1", "-I", CSRC, str(d / "plan.cpp"), "-o",
                    str(d / "plan")], check=True)

    def run(kv_heads, ratio, target, seqs, groups, dim=128):
        text = " ".join(map(str, [dim, kv_heads, ratio, target, len(seqs), len(groups)] + [x for s in seqs for x in s] +
                            [x for g in groups for x in g]))
        p = subprocess.run([str(d / "plan")], input=text, capture_output=True, text=True)
        assert p.returncode == 0, (p.returncode, text[:200])
        return [int(x) for x in p.stdout.split()]

    return run


def size(rng, most):
    return rng.choice([0, 1, rng.randint(0, 20), int(most ** rng.random()), int(most ** rng.random())])


@pytest.mark.parametrize("seed", range(60))
def test_bounds_hold(plan, seed):
    rng = random.Random(seed)
    for _ in range(20):
        most = rng.choice([1, 4, 40, 600, 9000])
        seqs = [(size(rng, most), size(rng, rng.choice([50, 3000, 1 << 20]))) for _ in range(rng.choice([1, 2, 9, 200]))]
        groups, left = [], len(seqs)
        while left and rng.random() < 0.8:
            n = rng.randint(0, left)
            groups.append((n, size(rng, 1 << 18)))
            left -= n
        units, most_units, parts, most_parts = plan(rng.choice([1, 2, 5, 8, 32]), rng.choice([1, 3, 4, 8, 32]),
                                                    rng.choice([256, 1024, 2048]), seqs, groups, rng.choice([64, 128, 256]))
        assert units <= most_units and parts <= most_parts, (seed, seqs[:5], groups[:5])


def test_edges(plan):
    assert plan(8, 4, 1024, [(0, 0)], [])[0] == 0
    assert plan(8, 4, 1024, [(1, 0)], [(1, 0)])[0] == 0
    units, most, _, _ = plan(1, 1, 1024, [(1, 2**31 - 1)], [])
    assert 512 <= units <= 1025 <= most + 1


def test_a_launch_without_groups_has_a_units_room_once(plan):
    units, most, parts, most_parts = plan(32, 1, 256, [(8192, 8192)], [])
    assert units <= most <= 2 * 256 + 32 * (64 + 4) and parts <= most_parts


@pytest.mark.parametrize("seed", range(20))
def test_bounds_hold_for_few_rows(plan, seed):
    """Where tiles are not full the bounds are closest."""
    rng = random.Random(1000 + seed)
    for _ in range(20):
        seqs = [(rng.choice([0, 1, 1, 2, 17, 64]), size(rng, 1 << 17)) for _ in range(rng.choice([1, 1, 2, 5]))]
        n = rng.randint(0, len(seqs))
        units, most_units, parts, most_parts = plan(rng.choice([1, 2, 8]), rng.choice([1, 1, 2, 4, 5]), 256, seqs,
                                                    [(n, size(rng, 1 << 17))] if rng.random() < 0.6 else [],
                                                    rng.choice([64, 128, 256]))
        assert units <= most_units and parts <= most_parts, (seed, seqs, n)


# Trees of drafts: items of few rows are cut for 256 units, the others for 480 where their chunks stay long.
TREE_BODY = BODY.replace("(uint32_t)target, (uint32_t)dim))", "256, (uint32_t)dim, target > 256 ? (uint32_t)target : 0))")
assert TREE_BODY.count("target > 256") == 1
# what an item of `rows` rows is cut into where all of its kind cost `cost`
CHUNK_BODY = r"""
#include <cstdio>
#include "prefix_plan.h"
int main() {
  unsigned long long rows, cost, dim;
  while (scanf("%llu %llu %llu", &rows, &cost, &dim) == 3)
    printf("%u %u\n", gleam::chunk_steps((uint32_t)rows, cost, 256, (uint32_t)dim, 480),
           gleam::chunk_steps((uint32_t)rows, cost, 256, (uint32_t)dim));
  return 0;
}
"""


def compiled(path, body):
    (path / "plan.cpp").write_text(body)
    subprocess.run([shutil.which("g++"), "-std=c++17", "-Wall", "-Werror", "-O1", "-I", CSRC, str(path / "plan.cpp"),
                    "-o", str(path / "plan")], check=True)

    def run(numbers):
        p = subprocess.run([str(path / "plan")], input=" ".join(map(str, numbers)), capture_output=True, text=True)
        assert p.returncode == 0, (p.returncode, numbers[:40])
        return [int(x) for x in p.stdout.split()]

    return run


@pytest.fixture(scope="module")
def trees(tmp_path_factory):
    run = compiled(tmp_path_factory.mktemp("trees"), TREE_BODY)
    return lambda kv_heads, ratio, seqs, groups, dim, target=480: run(
        [dim, kv_heads, ratio, target, len(seqs), len(groups)] + [x for s in seqs for x in s] +
        [x for g in groups for x in g])


def tile_cost(kv_heads, ratio, seqs):
    """Steps of all tiles of 128 rows, of sequences without groups."""
    return sum(-(-t * ratio // 128) * -(-own // 64) * kv_heads for t, own in seqs if t * ratio > 64)


# 9,120 steps and 9,129: 480 units would have 19 steps each, and 20
LONG_TREES = [[(33, own), (20, 33000), (9, 17000), (1, 5000), (2, 900)] for own in (638 * 64, 638 * 64 + 1)]


def test_where_trees_take_more_units(tmp_path, trees):
    chunks = compiled(tmp_path, CHUNK_BODY)
    below, above = (tile_cost(1, 32, seqs) for seqs in LONG_TREES)
    assert (below, above) == (480 * 19, 480 * 19 + 9)
    assert chunks([1056, below, 64, 1056, above, 64]) == [36, 36, 20, 36]
    assert chunks([64, above, 64, 16, above, 64]) == [36, 36] * 2  # few rows: never
    assert chunks([100, 1 << 40, 128]) == [0x7fffffff, 0x7fffffff]
    for dim in (64, 128, 256):  # what a chunk has at least, of few and of many rows
        assert chunks([64, 1, dim, 65, 1, dim]) == [2, 2, 512 // dim, 512 // dim]
    units = [trees(1, 32, seqs, [], 64)[0] for seqs in LONG_TREES]
    assert units[1] > units[0] + 100


@pytest.mark.parametrize("seed", range(60))
def test_bounds_hold_for_trees(trees, seed):
    """Launch and workspace of 480 units of each kind hold what is cut for 256 and 480, few and many rows mixed."""
    rng = random.Random(2000 + seed)
    long = 0
    for _ in range(20):
        kv_heads, ratio = rng.choice([1, 2, 5, 8, 32]), rng.choice([1, 3, 4, 8, 32])
        seqs = [(rng.choice([0, 1, 5, 17, 33, 64, 128, 300]), size(rng, rng.choice([500, 20000, 1 << 19])))
                for _ in range(rng.choice([1, 2, 4, 9, 100]))]
        groups, left = [], len(seqs)
        while left and rng.random() < 0.5:
            n = rng.randint(0, left)
            groups.append((n, size(rng, 1 << 17)))
            left -= n
        long += tile_cost(kv_heads, ratio, seqs) > 480 * 19
        units, most_units, parts, most_parts = trees(kv_heads, ratio, seqs, groups, rng.choice([64, 128]))
        assert units <= most_units and parts <= most_parts, (seed, seqs[:5], groups[:5])
    assert long


@pytest.mark.parametrize("over", [-9, -1, 0, 1, 9])
def test_bounds_hold_for_trees_next_to_the_border(trees, over):
    """One tile for each head: costs on both sides of where chunks of 480 units have 20 steps."""
    for kv_heads, tiles in ((1, 1), (1, 7), (4, 3), (8, 2), (5, 9)):
        steps = (480 * 19 + 1) // (kv_heads * tiles) + over
        seqs = [(128 * tiles, steps * 64)]
        for more in ([], [(1, 1 << 18)], [(16, 4096)] * 40):
            units, most_units, parts, most_parts = trees(kv_heads, 1, seqs + more, [], 128)
            assert units <= most_units and parts <= most_parts, (kv_heads, tiles, over, len(more))
