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
