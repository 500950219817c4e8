// How prefix_attention cuts its work, as plain arithmetic (a CPU test compiles this file by
// itself; on the GPU one workgroup runs it over the lengths it finds there).
//
// An item is a set of rows (one row for each token and query head of a key head) with the keys
// that all of them may see: a group's tokens with the group's prefix, or a sequence's tokens
// with its own keys. A sequence's item holds the group's prefix too ("joint") where sharing
// would save nothing: in a group of one, and where sequences have so many rows that each fills
// tiles of its own. Keys are walked in steps; an item's steps are cut into chunks, its rows into
// tiles, and a unit is one tile of one key head over one chunk. What a row gathers from several
// chunks, or from its group's item and its own, goes through partial results in the workspace
// and is joined afterwards.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define GLEAM_HD __host__ __device__ inline
#else
#define GLEAM_HD inline
#endif

namespace gleam {

constexpr uint32_t kStep = 64;        // keys in a step
constexpr uint32_t kFewRows = 16, kTileRows = 128;  // rows of a tile, of the two kinds
constexpr uint32_t kMostFew = 64;     // items of up to this many rows take tiles of the first kind
constexpr uint32_t kJointRows = 128;  // sequences of a group with this many rows on average keep to themselves
// Steps of the shortest chunks: one round of a workgroup's four waves; and of the second kind, whose
// partial results are 512 bytes a dim and unit, 256 keys of 128 dims, or as many bytes of others
// (64 rows behind 2,000 keys of 128 dims take 31 us with 4 steps, 35 with 8; 12 groups of 16 behind
// up to 4,096 of 64 dims 37 and 34).
constexpr uint32_t kMinFewSteps = 2;
GLEAM_HD uint32_t min_tile_steps(uint32_t head_dim) { return 512 / head_dim; }

struct PlanShape {  // what the host knows
  uint64_t n_tokens, n_seq, n_groups;
  uint32_t kv_heads, ratio;  // ratio: query heads per key head
  uint32_t target;           // units of each kind wanted (kUnits of the launch)
  uint32_t most_steps;       // of an item, from the widths of the page tables
  uint32_t head_dim;
};

GLEAM_HD uint64_t div_up(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

GLEAM_HD uint32_t steps_of(uint32_t keys) { return (keys + kStep - 1) / kStep; }

GLEAM_HD bool joint_group(uint64_t rows, uint64_t seqs) { return seqs <= 1 || rows >= kJointRows * seqs; }

GLEAM_HD bool few_rows(uint32_t rows) { return rows <= kMostFew; }
GLEAM_HD uint32_t tiles_of(uint32_t rows) {
  const uint32_t per = few_rows(rows) ? kFewRows : kTileRows;
  return (rows + per - 1) / per;
}

// What an item costs a key head: its tiles' steps.
GLEAM_HD uint64_t item_cost(uint32_t rows, uint32_t steps) { return (uint64_t)tiles_of(rows) * steps; }

// Steps of a chunk of an item of `rows` rows: no more than `target` chunks of all tiles of a kind
// together, apart from each tile's first. `cost`: of all items of the kind, all key heads.
GLEAM_HD uint32_t chunk_steps(uint32_t rows, uint64_t cost, uint32_t target, uint32_t head_dim) {
  const uint64_t c = div_up(cost, target), least = few_rows(rows) ? kMinFewSteps : min_tile_steps(head_dim);
  return c < least ? (uint32_t)least : c > 0x7fffffffu ? 0x7fffffffu : (uint32_t)c;
}

// Chunks of an item, and its own steps per chunk: as even as the count allows.
struct Cut {
  uint32_t chunks, per;
};
GLEAM_HD Cut cut_steps(uint32_t steps, uint32_t most) {
  Cut c{0, 1};
  if (steps == 0) return c;
  c.chunks = (steps + most - 1) / most;
  c.per = (steps + c.chunks - 1) / c.chunks;
  c.chunks = (steps + c.per - 1) / c.per;
  return c;
}

// The bounds that the launch and the workspace are sized by, from what the host knows.
//
// Units: sum of tiles * kv_heads * chunks, where chunks < steps / chunk_steps + 1, so at most
// 2 * target (one for each kind) + kv_heads * tiles, and at most kv_heads * tiles * most_steps /
// kMinFewSteps. Tiles: an item of n rows has at most n / kFewRows + 1 of them, and at most
// n / kTileRows + kMostFew / kFewRows, and a token's rows are in two items at most, its group's
// (if there are groups) and its sequence's.
GLEAM_HD uint64_t most_first_units(const PlanShape& s) {  // kv_heads * tiles
  const uint64_t rows = (s.n_groups ? 2 : 1) * s.n_tokens * s.ratio, items = s.n_groups + s.n_seq;
  const uint64_t few = items + rows / kFewRows, tile = kMostFew / kFewRows * items + rows / kTileRows;
  return s.kv_heads * (few < tile ? few : tile);
}
GLEAM_HD uint64_t most_units_any_width(const PlanShape& s) { return 2ull * s.target + most_first_units(s); }
GLEAM_HD uint64_t most_units(const PlanShape& s) {
  const uint64_t cuts = most_first_units(s) * div_up(s.most_steps, kMinFewSteps), any = most_units_any_width(s);
  return cuts < any ? cuts : any;
}

// Rows of partial results: an item that is cut, or shares its rows with another, has
// rows * kv_heads * chunks. Shared: groups that are not joint have fewer than kJointRows rows a
// sequence, in two items, for their first chunks. Cut: chunks >= 2 makes chunks <= 2 * steps /
// chunk_steps, and an item's rows <= the rows of a tile * tiles, so 2 * target of the rows of a
// tile at most for each kind. A tile has no more rows than all tokens have, and of the second kind
// there is none where those are few.
GLEAM_HD uint64_t most_partials(const PlanShape& s) {
  const uint64_t rows = s.n_tokens * s.ratio, apart = kJointRows * s.n_seq;
  const uint64_t shared = s.n_groups ? 2 * (rows < apart ? rows : apart) * s.kv_heads : 0;
  const uint64_t few = rows < kFewRows ? rows : kFewRows;
  const uint64_t tile = rows <= kMostFew ? 0 : rows < kTileRows ? rows : kTileRows;
  return shared + 2 * (few + tile) * s.target;
}

}  // namespace gleam
