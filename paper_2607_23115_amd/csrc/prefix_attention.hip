// Attention of a ragged batch over a paged key/value cache, in which groups of sequences share a
// prefix: prefix keys and values are read and scored once for all rows of a group.
//
// A row's result over any set of keys is (m, l, o): m the largest score, l = sum exp(score - m),
// o = sum exp(score - m) v. Two sets join as m = max, l and o weighted by exp(their m - m), so
// keys can be walked in any order and pieces: one pass over the keys with running m, l, o; long
// walks cut into chunks for several workgroups; the shared prefix and a sequence's own keys as
// separate pieces of one row. Scores are kept times log2(e), so that every exponential is one
// hardware exp2.
//
// attend_kernel takes a unit per workgroup, join_kernel joins the pieces. The lengths found on the
// device are cut into units (prefix_plan.h) by plan_kernel, or, in a batch of up to 63 items, by
// every wave of attend_kernel for itself, an item a lane: that takes about a microsecond, a launch
// and the wait for it several.
//
// A unit is 16 rows of one key head. Four waves take turns at 32 keys each, straight from memory
// to registers in the layouts of v_mfma_f32_16x16x32: nothing is exchanged between lanes but the
// maximum over a wave's keys.
//   scores  S^T = K Q^T, a product for each 16 keys. A lane holds, as K's row operand, 8 dims of
//           key (lane % 16), and gets the scores of row (lane % 16) with keys 4 g .. 4 g + 3, g =
//           lane / 16.
//   output  O^T = V^T P^T over 32 keys at once. The order of keys within a product is free: taking
//           keys {4g..4g+3} of the first 16 and of the second 16 as the eight that lane group g
//           brings makes its own scores, once exponentiated, P's operand as they are. As V's
//           operand a lane holds those 8 keys' dims (lane % 16) * D/16 .. + D/16, loaded row by
//           row and transposed within the lane.
// With few rows this is bound by reading the keys and values once: one token of 32 heads behind
// 131,071 keys of 8 heads of 128 takes 85 us (6.3 TB/s; a plain read reaches 7.1), the join 5 more. 64
// sequences of 8,192 keys, nothing shared, take 366 us, 5.9 TB/s.
// Items of more than 64 rows take units of 128 rows (attend_tile).

#include <type_traits>

#include "kv_pages.h"
#include "launch_shape.h"
#include "prefix_plan.h"

namespace gleam {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kPlanThreads = 1024;
constexpr float kRise = 8.f;  // log2
// The exponentials' reference is 2^up below the score that it follows: 16 bits of fp16 hold them from
// 2^-25 on, and without it the many small ones of a long history would be in a row's sum, but not in its
// output (a key and 65,536 others 2^25 below it: 0.2% of the output). They go up to 2^15 that way. bf16
// reaches down to 2^-133, and its values so far up that their sums need the room.
template <class T> constexpr float kUp = std::is_same_v<T, Fp16> ? 7.f : 0.f;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr uint64_t kMostSeq = 1ull << 20;
constexpr uint64_t kPassing = 128ull << 20;  // bytes of an item's keys and values
constexpr uint32_t kWideJoin = 256;    // up to this many rows are joined by a workgroup each
constexpr uint32_t kMostJoins = 2048;  // workgroups of the others: those that the GPU holds at once
// Units wanted of each kind: one a CU, chosen by measurement. A CU holds two (of heads of 256 one), but
// with 512 an item is cut into twice the pieces: 1.6% slower over twelve cases and fourteen drawn ones, 128
// sequences behind 8,192 keys 70 us for 58.
constexpr uint32_t kUnits = 256;

struct Item {
  uint32_t token_first, tokens;  // rows: tokens * ratio
  uint32_t prefix_row, prefix_keys;  // the shared pages' row of the table and how many keys; 0: none
  uint32_t own_row, own_keys;        // the sequence's own
  uint32_t chunks, per;              // chunks and steps of each; 0: no keys at all
  uint32_t tile_first, few_first;    // units of full tiles and of few rows before it: its own first
  uint32_t part_first;               // the first row of partial results
  uint32_t partial;                  // results go to the workspace
  uint32_t pad[4];
};

struct PlanHeader {
  uint32_t tiles, fews;  // units of the two kinds
  uint32_t joins;        // some row needs join_kernel
};

struct Ws {  // device addresses within the workspace
  PlanHeader* head;
  int32_t* q_first;      // [n_seq + 1] as used: clamped, non-decreasing
  int32_t* group_first;  // [n_groups + 1]
  int32_t* seq_group;    // [n_seq], -1: none
  uint32_t* tile_first;  // [n_groups + n_seq], of the items
  uint32_t* few_first;
  Item* items;           // groups, then sequences
  float* part_o;         // [partials][head_dim]
  float* part_ml;        // [partials][2]: m (log2), l
  size_t bytes;
};

struct AttendArgs {
  const uint8_t* q;
  int64_t q_token, q_head;  // bytes
  const uint8_t* k;
  const uint8_t* v;
  int64_t k_page, k_place, k_head, v_page, v_place, v_head;  // bytes
  const int32_t* q_first;
  const int32_t* own_pages;
  const int32_t* own_len;
  const int32_t* group_first;
  const int32_t* prefix_pages;
  const int32_t* prefix_len;
  uint32_t n_tokens, n_seq, n_groups, own_width, prefix_width;
  uint32_t q_heads, kv_heads, ratio, page_log2, n_pages, target, head_dim;
  float scale_log2;
  uint8_t* out;
  float* lse;
  Ws ws;
};

Ws ws_at(uint8_t* base, const PlanShape& s, uint32_t head_dim) {
  Ws w{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    uint8_t* p = base + at;
    at += (bytes + 255) & ~(size_t)255;
    return p;
  };
  const uint64_t items = s.n_groups + s.n_seq, partials = most_partials(s);
  w.head = reinterpret_cast<PlanHeader*>(take(sizeof(PlanHeader)));
  w.q_first = reinterpret_cast<int32_t*>(take((s.n_seq + 1) * 4));
  w.group_first = reinterpret_cast<int32_t*>(take((s.n_groups + 1) * 4));
  w.seq_group = reinterpret_cast<int32_t*>(take(s.n_seq * 4));
  w.tile_first = reinterpret_cast<uint32_t*>(take(items * 4));
  w.few_first = reinterpret_cast<uint32_t*>(take(items * 4));
  w.items = reinterpret_cast<Item*>(take(items * sizeof(Item)));
  w.part_o = reinterpret_cast<float*>(take(partials * head_dim * 4));
  w.part_ml = reinterpret_cast<float*>(take(partials * 8));
  w.bytes = at;
  return w;
}

// --------------------------------------------------------------------------------------- //
// plan
// --------------------------------------------------------------------------------------- //
struct SumOp {
  template <class V> __device__ V operator()(V a, V b) const { return a + b; }
};
struct MaxOp {
  template <class V> __device__ V operator()(V a, V b) const { return a > b ? a : b; }
};

// The value that a DPP control brings to each lane, `none` where it brings nothing.
template <int kCtrl, int kRows>
__device__ inline uint32_t dpp(uint32_t v, uint32_t none) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)none, (int)v, kCtrl, kRows, 0xf, false);
}
template <int kCtrl, int kRows>
__device__ inline int32_t dpp(int32_t v, int32_t none) {
  return __builtin_amdgcn_update_dpp(none, v, kCtrl, kRows, 0xf, false);
}
template <int kCtrl, int kRows>
__device__ inline uint64_t dpp(uint64_t v, uint64_t none) {
  return (uint64_t)dpp<kCtrl, kRows>((uint32_t)(v >> 32), (uint32_t)(none >> 32)) << 32 |
         dpp<kCtrl, kRows>((uint32_t)v, (uint32_t)none);
}

// Inclusive scan over a wave of values that 0 leaves as they are: shifts by 1, 2, 4 and 8 within
// rows of 16 lanes, then the last lanes of rows 0 and 2 to the rows after them, then lane 31 to
// the upper half.
template <class V, class Op>
__device__ V wave_scan(V v, Op op) {
  v = op(dpp<0x111, 0xf>(v, (V)0), v);
  v = op(dpp<0x112, 0xf>(v, (V)0), v);
  v = op(dpp<0x114, 0xf>(v, (V)0), v);
  v = op(dpp<0x118, 0xf>(v, (V)0), v);
  v = op(dpp<0x142, 0xa>(v, (V)0), v);
  v = op(dpp<0x143, 0xc>(v, (V)0), v);
  return v;
}

// The same over the workgroup, of kN values at once (two barriers); every thread calls it. `total`
// gets the last values.
template <int kN, class V, class Op>
__device__ void block_scan(V (&v)[kN], V (&total)[kN], V (*lds)[kN], Op op) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < kN; ++i) v[i] = wave_scan(v[i], op);
  if (lane == 63) {
#pragma unroll
    for (int i = 0; i < kN; ++i) lds[wave][i] = v[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    V all = lds[0][i];
    for (int w = 1; w < (int)(blockDim.x >> 6); ++w) {
      if (w == wave) v[i] = op(all, v[i]);
      all = op(all, lds[w][i]);
    }
    total[i] = all;
  }
  __syncthreads();
}

__device__ inline int32_t clamp_to(int32_t v, int32_t most) { return v < 0 ? 0 : v > most ? most : v; }

// How many keys a length means: none in a cache without pages.
__device__ inline uint32_t clamp_keys(const AttendArgs& a, int32_t n, uint32_t width) {
  return a.n_pages ? (uint32_t)clamp_to(n, (int32_t)(width << a.page_log2)) : 0;
}

// Item i without its cut. q(i), g(i): the offsets, already tidy; own(s), prefix(g): lengths as
// given; group_of(s): -1 for none. All lanes call them, with indexes in range.
template <class Q, class G, class Own, class Prefix, class GroupOf>
__device__ Item make_item(const AttendArgs& a, uint32_t i, const Q& q, const G& g, const Own& own,
                          const Prefix& prefix, const GroupOf& group_of) {
  const bool is_group = i < a.n_groups;
  const uint32_t s = is_group || i >= a.n_groups + a.n_seq ? 0 : i - a.n_groups;
  const uint32_t t0 = (uint32_t)q(s), t1 = (uint32_t)q(s + 1);
  const uint32_t own_keys = clamp_keys(a, own(s), a.own_width);
  uint32_t shared = 0, g0 = 0, g1 = 0, row = 0;  // the group's prefix
  if (a.n_groups) {
    const int32_t of_seq = group_of(s), in = is_group ? (int32_t)i : of_seq;
    row = in < 0 ? 0 : (uint32_t)in;
    const uint32_t s0 = (uint32_t)g(row), s1 = (uint32_t)g(row + 1);
    g0 = (uint32_t)q(s0);
    g1 = (uint32_t)q(s1);
    const uint32_t keys = clamp_keys(a, prefix(row), a.prefix_width);
    if (in >= 0) shared = keys;
    // keys that the group's item has, and the sequence's has not
    if (joint_group((uint64_t)(g1 - g0) * a.ratio, s1 - s0) == is_group) {
      if (is_group) shared = 0;
      else row = ~0u;
    }
  }
  Item it{};
  if (is_group) {
    it.token_first = g0;
    it.tokens = g1 - g0;
    it.prefix_row = row;
    it.prefix_keys = shared;
    it.partial = 1;
  } else {
    it.token_first = t0;
    it.tokens = t1 - t0;
    it.own_row = s;
    it.own_keys = own_keys;
    it.partial = row == ~0u && shared > 0;
    it.prefix_row = row == ~0u ? 0 : row;
    it.prefix_keys = row == ~0u ? 0 : shared;
  }
  return it;
}

__device__ inline uint32_t item_steps(const Item& it) {
  return it.tokens ? steps_of(it.prefix_keys) + steps_of(it.own_keys) : 0;
}

// What the items of the two kinds cost together.
struct Costs {
  uint64_t tiles, fews;
};
__device__ inline Costs item_costs(const AttendArgs& a, const Item& it) {
  const uint32_t rows = it.tokens * a.ratio;
  const uint64_t cost = item_cost(rows, item_steps(it)) * a.kv_heads;
  return few_rows(rows) ? Costs{0, cost} : Costs{cost, 0};
}

// What an item takes, once cut (cost: all items'): units of the two kinds, rows of partial results.
// The sums over all items stay below 2^32 (most_units, most_partials).
struct Takes {
  uint32_t tiles, fews, parts;
};
__device__ inline Takes cut_item(const AttendArgs& a, Item& it, const Costs& cost) {
  const uint32_t rows = it.tokens * a.ratio;
  const Cut cut = cut_steps(item_steps(it), chunk_steps(rows, few_rows(rows) ? cost.fews : cost.tiles, a.target,
                                                    a.head_dim));
  it.chunks = cut.chunks;
  it.per = cut.per;
  if (cut.chunks > 1) it.partial = 1;
  const uint32_t units = tiles_of(rows) * a.kv_heads * cut.chunks;
  return {few_rows(rows) ? 0 : units, few_rows(rows) ? units : 0, it.partial ? it.tokens * a.q_heads * cut.chunks : 0};
}

// The plan of a batch of up to 63 items as every wave has it: item i in lane i.
constexpr uint32_t kWaveItems = 63;

struct WavePlan {
  Item it;          // of the lane
  int32_t q;        // tidy offset, of the lane
  int32_t group;    // of sequence `lane`
  uint32_t tiles, fews, joins;
};

__device__ WavePlan plan_in_wave(const AttendArgs& a) {
  const uint32_t lane = threadIdx.x & 63, n_items = a.n_groups + a.n_seq;
  WavePlan w;
  int32_t q = lane <= a.n_seq ? a.q_first[lane] : (int32_t)a.n_tokens;
  int32_t g = a.n_groups && lane <= a.n_groups ? a.group_first[lane] : (int32_t)a.n_seq;
  const int32_t own = lane < a.n_seq ? a.own_len[lane] : 0;
  const int32_t prefix = lane < a.n_groups ? a.prefix_len[lane] : 0;
  q = wave_scan(clamp_to(q, (int32_t)a.n_tokens), MaxOp());
  w.q = q;
  w.group = -1;
  if (a.n_groups) {
    g = wave_scan(clamp_to(g, (int32_t)a.n_seq), MaxOp());
    // the last group that starts at or before the sequence, if it has not ended there
    for (uint32_t i = 0; i < a.n_groups; ++i) {
      const int32_t from = __builtin_amdgcn_readlane(g, (int)i), to = __builtin_amdgcn_readlane(g, (int)i + 1);
      if ((int32_t)lane >= from && (int32_t)lane < to) w.group = (int32_t)i;
    }
  }
  auto of = [](int32_t v) { return [v](uint32_t i) { return __shfl(v, (int)i, 64); }; };
  w.it = make_item(a, lane, of(q), of(g), of(own), of(prefix), of(w.group));
  if (lane >= n_items) w.it = Item{};
  Costs cost = item_costs(a, w.it);
  cost.tiles = __shfl(wave_scan(cost.tiles, SumOp()), 63, 64);
  cost.fews = __shfl(wave_scan(cost.fews, SumOp()), 63, 64);
  const Takes mine = cut_item(a, w.it, cost);
  const uint32_t tiles = wave_scan(mine.tiles, SumOp()), fews = wave_scan(mine.fews, SumOp());
  w.it.tile_first = tiles - mine.tiles;
  w.it.few_first = fews - mine.fews;
  w.it.part_first = wave_scan(mine.parts, SumOp()) - mine.parts;
  w.tiles = (uint32_t)__builtin_amdgcn_readlane((int)tiles, 63);
  w.fews = (uint32_t)__builtin_amdgcn_readlane((int)fews, 63);
  const bool empty = lane >= a.n_groups && w.it.tokens && item_steps(w.it) == 0;
  w.joins = __any(empty || mine.parts != 0) || __shfl(q, 0, 64) > 0 ||
            __shfl(q, (int)a.n_seq, 64) < (int32_t)a.n_tokens;
  return w;
}

// For join_kernel: what plan_kernel leaves behind. By one wave.
__device__ inline void write_plan(const AttendArgs& a, const WavePlan& plan) {
  const Ws& w = a.ws;
  const uint32_t lane = threadIdx.x & 63;
  if (lane <= a.n_seq) w.q_first[lane] = plan.q;
  if (lane < a.n_seq) w.seq_group[lane] = plan.group;
  if (lane < a.n_groups + a.n_seq) w.items[lane] = plan.it;
  if (lane == 0) w.head->joins = plan.joins;
}

// Of a value that is the same in all lanes: kept in a scalar register, branches on it not masked.
__device__ inline uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// Lane i's item, in all lanes.
__device__ inline Item item_of_lane(const Item& it, uint32_t i) {
  auto get = [i](uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, (int)i); };
  Item r{};
  r.token_first = get(it.token_first);
  r.tokens = get(it.tokens);
  r.prefix_row = get(it.prefix_row);
  r.prefix_keys = get(it.prefix_keys);
  r.own_row = get(it.own_row);
  r.own_keys = get(it.own_keys);
  r.chunks = get(it.chunks);
  r.per = get(it.per);
  r.tile_first = get(it.tile_first);
  r.few_first = get(it.few_first);
  r.part_first = get(it.part_first);
  r.partial = get(it.partial);
  return r;
}

// One workgroup, whose time is that of its loads and seven barriers: 4.3 us for 65 items, 6.2 for
// 204. Offsets of up to this many sequences and groups are kept in LDS, of more in the workspace.
constexpr uint32_t kPlanLds = 4096;

__global__ __launch_bounds__(kPlanThreads) void plan_kernel(AttendArgs a) {
  __shared__ uint64_t lds_costs[kPlanThreads / 64][2];
  __shared__ uint32_t lds_takes[kPlanThreads / 64][4];
  __shared__ int32_t lds_tidy[kPlanThreads / 64][2];
  __shared__ int32_t lds_q[kPlanLds + 1], lds_g[kPlanLds + 1];
  const Ws& w = a.ws;
  const uint32_t n_items = a.n_groups + a.n_seq, threads = blockDim.x;
  int32_t* const q = a.n_seq <= kPlanLds ? lds_q : w.q_first;
  int32_t* const g = a.n_groups <= kPlanLds ? lds_g : w.group_first;

  // the offsets as non-decreasing values in their ranges
  const uint32_t offsets = a.n_groups > a.n_seq ? a.n_groups : a.n_seq;
  int32_t carry[2] = {0, 0};
  for (uint32_t i0 = 0; i0 <= offsets; i0 += threads) {
    const uint32_t i = i0 + threadIdx.x;
    const bool has_g = a.n_groups && i <= a.n_groups;
    int32_t v[2] = {clamp_to(i <= a.n_seq ? a.q_first[i] : 0, (int32_t)a.n_tokens),
                    clamp_to(has_g ? a.group_first[i] : 0, (int32_t)a.n_seq)};
    int32_t total[2];
    block_scan(v, total, lds_tidy, MaxOp());
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      v[c] = v[c] > carry[c] ? v[c] : carry[c];
      carry[c] = carry[c] > total[c] ? carry[c] : total[c];
    }
    if (i <= a.n_seq) w.q_first[i] = q[i] = v[0];
    if (has_g) g[i] = v[1];
  }
  __syncthreads();
  auto group_of = [&](uint32_t s) {
    if ((int32_t)s < g[0] || (int32_t)s >= g[a.n_groups]) return -1;
    uint32_t lo = 0, hi = a.n_groups;  // g[lo] <= s < g[hi]
    while (hi - lo > 1) {
      const uint32_t mid = (lo + hi) / 2;
      if (g[mid] <= (int32_t)s) lo = mid;
      else hi = mid;
    }
    return (int32_t)lo;
  };
  auto of = [](const int32_t* v) { return [v](uint32_t i) { return v[i]; }; };

  // the items without their cuts, and the cost of all
  uint64_t costs[2] = {0, 0}, all_costs[2];
  uint32_t joins = q[0] > 0 || q[a.n_seq] < (int32_t)a.n_tokens;
  Item first{};  // of the thread; those of later rounds go through the workspace
  for (uint32_t i = threadIdx.x; i < n_items; i += threads) {
    Item it = make_item(a, i, of(q), of(g), of(a.own_len), of(a.prefix_len), group_of);
    const Costs c = item_costs(a, it);
    costs[0] += c.tiles;
    costs[1] += c.fews;
    if (i >= a.n_groups && it.tokens && item_steps(it) == 0) joins = 1;
    if (i < threads) first = it;
    else w.items[i] = it;
    if (a.n_groups && i >= a.n_groups) w.seq_group[i - a.n_groups] = group_of(i - a.n_groups);
  }
  block_scan(costs, all_costs, lds_costs, SumOp());

  // chunks, units and partial rows
  uint32_t before[4] = {0, 0, 0, 0};
  for (uint32_t i0 = 0; i0 < n_items; i0 += threads) {
    const uint32_t i = i0 + threadIdx.x;
    Item it = first;
    if (i0 > 0) {
      it = Item{};
      if (i < n_items) it = w.items[i];
    }
    const Takes mine = cut_item(a, it, Costs{all_costs[0], all_costs[1]});
    uint32_t sum[4] = {mine.tiles, mine.fews, mine.parts, joins | (mine.parts != 0)}, total[4];
    joins = 0;
    block_scan(sum, total, lds_takes, SumOp());
    it.tile_first = before[0] + sum[0] - mine.tiles;
    it.few_first = before[1] + sum[1] - mine.fews;
    it.part_first = before[2] + sum[2] - mine.parts;
    if (i < n_items) {
      w.items[i] = it;
      w.tile_first[i] = it.tile_first;
      w.few_first[i] = it.few_first;
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) before[c] += total[c];
  }
  if (threadIdx.x == 0) {
    w.head->tiles = before[0];
    w.head->fews = before[1];
    w.head->joins = before[3];
  }
}

// The last i of [0, n) with first[i] <= x, found by a wave: 64 probes a round. first is
// non-decreasing and first[0] <= x; x is the same in all lanes.
template <class V>
__device__ uint32_t wave_search(const V* first, uint32_t n, V x) {
  const uint32_t lane = threadIdx.x & 63;
  uint32_t lo = 0, hi = n;
  while (hi - lo > 1) {
    const uint32_t stride = (hi - lo + 63) / 64;
    const uint32_t at = lo + lane * stride;
    const uint64_t le = __ballot(at < hi && first[at < hi ? at : lo] <= x);
    const uint32_t last = 63 - __clzll((long long)le);
    const uint32_t from = lo + last * stride;
    const uint32_t to = from + stride;
    lo = from;
    hi = to < hi ? to : hi;
  }
  return lo;
}

// --------------------------------------------------------------------------------------- //
// attend
// --------------------------------------------------------------------------------------- //
template <class T> struct Mfma;
template <> struct Mfma<Fp16> {
  static __device__ f32x4 run(f16x8 a, f16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
  }
};
template <> struct Mfma<Bf16> {
  static __device__ f32x4 run(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
  }
};

union Pack8 {
  u32x4v u;
  f16x8 h;
  bf16x8 b;
};
__device__ inline void put(Pack8& p, int i, float x, Fp16) { p.h[i] = (_Float16)x; }
__device__ inline void put(Pack8& p, int i, float x, Bf16) { p.b[i] = (__bf16)x; }
__device__ inline f16x8 get(const Pack8& p, Fp16) { return p.h; }
__device__ inline bf16x8 get(const Pack8& p, Bf16) { return p.b; }

// An infinite or NaN value of a key that some rows of a tile may not see would reach them as
// 0 * infinity. Where a tile has such keys, its values are looked at, the infinite and NaN ones
// are taken as 0 in the products, and add_special adds them at the end to the rows that see them.

// Bit 15 of each half of the result: the exponent of the 16-bit value there is all ones (the
// lowest exponent bit added to it carries into the sign's place).
template <class T>
__device__ inline uint32_t special_bits(uint32_t x) {
  constexpr uint32_t low = T::kExp & (0u - T::kExp);
  return ((x & (T::kExp * 0x10001u)) + low * 0x10001u) & 0x80008000u;
}
template <class T>
__device__ inline uint32_t clear_special(uint32_t x) {
  return x & ~((special_bits<T>(x) >> 15) * 0xffffu);
}

// A number that no cache has a page of.
constexpr uint32_t kNoPage = ~0u;

// The page of an item's key `key`, of `keys`.
__device__ inline uint32_t page_at(const AttendArgs& a, const int32_t* pages, uint32_t key, uint32_t keys) {
  return key < keys ? (uint32_t)pages[key >> a.page_log2] : kNoPage;
}

// Where the keys from `key` on are, up to the 16 that lie in its page (key a multiple of 8; fewer
// than 16 are used where it is not one of 16).
struct Keys16 {
  const uint8_t* k;
  const uint8_t* v;
  uint32_t n;  // how many of them exist
};
__device__ inline Keys16 keys16(const AttendArgs& a, uint32_t page, uint32_t key, uint32_t keys, uint32_t head) {
  Keys16 t{a.k, a.v, 0};
  if (page >= a.n_pages || key >= keys) return t;
  const uint32_t place = key & ((1u << a.page_log2) - 1);
  t.k = a.k + (int64_t)page * a.k_page + (int64_t)place * a.k_place + (int64_t)head * a.k_head;
  t.v = a.v + (int64_t)page * a.v_page + (int64_t)place * a.v_place + (int64_t)head * a.v_head;
  t.n = keys - key < 16 ? keys - key : 16;
  return t;
}

// What is at a base that is the same in all lanes and the lane's own offset, added by the load;
// kOnce: what nobody reads again soon is not kept in the caches.
template <class V, bool kOnce = false>
__device__ inline V load_at(const uint8_t* base, uint32_t offset) {
  uint64_t x = reinterpret_cast<uint64_t>(base);
  asm("" : "+s"(x));  // kept apart from the offset
  typedef const __attribute__((address_space(1))) uint8_t* Global;
  const auto* p = reinterpret_cast<const __attribute__((address_space(1))) V*>(reinterpret_cast<Global>(x) + offset);
  return kOnce ? __builtin_nontemporal_load(p) : *p;
}

// Calls add(i, value) for kN values, with 0 in the place of finite ones.
template <class T, int kN, class Add>
__device__ inline void add_special(const uint8_t* v, const Add& add) {
#pragma unroll
  for (int i = 0; i < kN; i += 4) {
    const u32x2v x = *reinterpret_cast<const u32x2v*>(v + 2 * i);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint32_t bits = (x[c >> 1] >> (16 * (c & 1))) & 0xffffu;
      // as 32-bit bits, 0 for a finite value; no branches, there are many of these
      const uint32_t wide = T::kExp == 0x7f80u ? bits << 16
                                               : (bits & 0x8000u) << 16 | 0x7f800000u | (bits & 0x3ffu) << 13;
      add(i + c, __uint_as_float(wide & (0u - (special_bits<T>(bits) >> 15))));
    }
  }
}

// max and sum of a lane's value and that of the lane 32 away, max also of the lane 16 away
__device__ inline float max_rows(float x) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// A sum that small terms are added to for long: `lost` gathers what each addition rounds off.
struct Sum {
  float sum = 0.f, lost = 0.f;
  __device__ void add(float x) {
    const float t = sum + x;
    lost += x - (t - sum);
    sum = t;
  }
  __device__ void scale(float f) {
    sum *= f;
    lost *= f;
  }
  __device__ float value() const { return sum + lost; }
};

// The sum of kN values, in pairs.
template <int kN>
__device__ inline float sum_of(const float* x) {
  if constexpr (kN == 1) return x[0];
  else return sum_of<kN / 2>(x) + sum_of<kN / 2>(x + kN / 2);
}

// A unit, as its workgroup finds it.
struct Unit {
  Item it;
  uint32_t head, chunk, tile;
};

// 16 rows, the waves taking turns at the keys.
template <class T, int D>
__device__ __forceinline__ void attend_few(const AttendArgs& a, const Unit& unit, char* lds) {
  typedef typename T::scalar scalar;
  constexpr int kDims = D / 16;       // dims a lane brings of a value row
  constexpr int kWords = kDims / 2;   // as dwords
  constexpr int kKMfma = D / 32;      // products over a key's dims
  constexpr int kPad = D + 4;         // row of the workgroup's partial outputs in LDS
  typedef float RowsO[kFewRows][kPad];
  typedef float Rows[kFewRows];
  RowsO* const lds_o = reinterpret_cast<RowsO*>(lds);
  Rows* const lds_m = reinterpret_cast<Rows*>(lds + kWaves * sizeof(RowsO));
  Rows* const lds_l = lds_m + kWaves;
  const Item& it = unit.it;
  const uint32_t head = unit.head, chunk = unit.chunk, tile = unit.tile;
  const uint32_t rows = it.tokens * a.ratio;
  const Ws& w = a.ws;

  const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const uint32_t n = lane & 15, g = lane >> 4;
  const uint32_t row = tile * kFewRows + n;
  const bool row_live = row < rows;
  const uint32_t token = it.token_first + (row_live ? row / a.ratio : 0);
  const uint32_t q_head = head * a.ratio + (row_live ? row % a.ratio : 0);

  // keys of the sequence's own that the row sees; the fewest of the tile's rows
  const int64_t behind = (int64_t)it.own_keys - it.tokens + 1;
  const int64_t sees = behind + (row_live ? row / a.ratio : 0);
  const uint32_t own_seen = sees < 0 ? 0 : (uint32_t)sees;
  const int64_t fewest = behind + tile * kFewRows / a.ratio;
  const uint32_t own_least = fewest < 0 ? 0 : (uint32_t)fewest;
  uint32_t last_row = tile * kFewRows + kFewRows - 1;
  if (last_row >= rows) last_row = rows - 1;
  const int64_t furthest = behind + last_row / a.ratio;
  const uint32_t own_most = furthest < 0 ? 0 : furthest > it.own_keys ? it.own_keys : (uint32_t)furthest;

  Pack8 q[kKMfma];
#pragma unroll
  for (int i = 0; i < kKMfma; ++i) {
    q[i].u = (u32x4v)0u;
    if (row_live)
      q[i].u = *reinterpret_cast<const u32x4v*>(a.q + (int64_t)token * a.q_token + (int64_t)q_head * a.q_head +
                                                (i * 32 + g * 8) * 2);
  }

  const int32_t* const prefix_pages = a.prefix_pages + (uint64_t)it.prefix_row * a.prefix_width;
  const int32_t* const own_pages = a.own_pages + (uint64_t)it.own_row * a.own_width;
  const uint32_t prefix_halves = 2 * steps_of(it.prefix_keys);
  const uint32_t all_halves = prefix_halves + (own_most + 31) / 32;
  uint32_t end = 2 * (chunk + 1) * it.per;
  if (end > all_halves) end = all_halves;

  bool special = false;
  float m = -INFINITY;
  Sum l_sum;
  f32x4 o[kDims];
#pragma unroll
  for (int j = 0; j < kDims; ++j) o[j] = (f32x4)0.f;

  const uint32_t begin = 2 * chunk * it.per + wave;
  auto keys_of = [&](uint32_t half) { return half < prefix_halves ? it.prefix_keys : it.own_keys; };
  auto key_of = [&](uint32_t half) { return 32 * (half < prefix_halves ? half : half - prefix_halves); };
  // whose infinite and NaN values are taken out and added at the end: a half with an own key that some
  // row of the tile must not see (keys that do not exist are no reason, their values are set to 0)
  auto looked_at = [&](uint32_t half) { return half >= prefix_halves && key_of(half) + 32 > own_least; };

  // Pages ahead: lane 2 i has that of the first 16 keys of the wave's i-th half from page_half on,
  // lane 2 i + 1 that of the others. A half's keys wait for no look-up of their own.
  auto pages_from = [&](uint32_t half) {
    half += (lane >> 1) * kWaves;
    if (half >= end) return kNoPage;
    return page_at(a, half < prefix_halves ? prefix_pages : own_pages, key_of(half) + 16 * (lane & 1), keys_of(half));
  };
  uint32_t page_half = begin, pages = pages_from(begin);

  // The keys and values of two halves: those of the next are on their way during the products. All
  // places of 16 are loaded, whether keys or not: they lie in one page, and in the cache's first
  // where there is no page (without pages there are no keys, without keys no halves). Keys that are
  // none are masked, and the values in their place set to 0.
  u32x4v kk[2][2][kKMfma];
  uint32_t vv[2][8][kWords], exist[2][2];
  const uint32_t k_off = n * (uint32_t)a.k_place + g * 16;
  uint32_t v_off[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v_off[e] = (4 * g + e) * (uint32_t)a.v_place + n * (kDims * 2);
  auto load_tile = [&](const Keys16& t, auto set_, int b, auto once_) {
    constexpr int set = decltype(set_)::value;
    constexpr bool kOnce = decltype(once_)::value;
#pragma unroll
    for (int i = 0; i < kKMfma; ++i) kk[set][b][i] = load_at<u32x4v, kOnce>(t.k + i * 64, k_off);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      typedef std::conditional_t<kDims == 4, u32x2v, u32x4v> Part;
      constexpr int kPart = sizeof(Part) / 4;
#pragma unroll
      for (int c = 0; c < kWords / kPart; ++c) {
        const Part x = load_at<Part, kOnce>(t.v + 4 * kPart * c, v_off[e]);
#pragma unroll
        for (int d = 0; d < kPart; ++d) vv[set][4 * b + e][kPart * c + d] = x[d];
      }
    }
  };
  // An item's keys and values that one tile reads, and that are too many for the caches to have at the
  // next call, are not kept there (one token of 8 key heads: behind 131,072 keys 90 us, 102 where they
  // are; behind 32,768 31.0 and 30.5). What the rest of the batch reads is not looked at.
  const bool once = rows <= kFewRows && ((uint64_t)it.prefix_keys + it.own_keys) * a.kv_heads * (4 * D) >= kPassing;
  auto load_half = [&](uint32_t half, auto set_) {
    constexpr int set = decltype(set_)::value;
    if (half - page_half >= 32 * kWaves) {
      page_half = half;
      pages = pages_from(half);
    }
    const uint32_t at = (half - page_half) / kWaves * 2;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint32_t page = (uint32_t)__builtin_amdgcn_readlane((int)pages, (int)(at + b));
      const Keys16 t = keys16(a, page, key_of(half) + 16 * b, keys_of(half), head);
      exist[set][b] = t.n;
      if (once) {
        asm volatile("");  // the two kinds of loads are not to be merged into one
        load_tile(t, set_, b, std::true_type());
        asm volatile("");
      } else {
        load_tile(t, set_, b, std::false_type());
      }
    }
  };

  auto do_half = [&](uint32_t half, auto set_) {
    constexpr int set = decltype(set_)::value;
    typedef std::integral_constant<int, 1 - set> Other;
    if (half + kWaves < end) load_half(half + kWaves, Other());
    const bool shared = half < prefix_halves;
    const uint32_t key = key_of(half);
    f32x4 s[2] = {(f32x4)0.f, (f32x4)0.f};
#pragma unroll
    for (int i = 0; i < kKMfma; ++i) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        Pack8 k;
        k.u = kk[set][b][i];
        s[b] = Mfma<T>::run(get(k, T()), get(q[i], T()), s[b]);
      }
    }
    // whether some row of the tile must not see some key of these 32
    const uint32_t least = shared ? it.prefix_keys : own_least;
    const bool masked = key + 32 > least || exist[set][0] + exist[set][1] < 32;
    const uint32_t seen = shared ? it.prefix_keys : own_seen;
    float x[8], top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = s[e >> 2][e & 3] * a.scale_log2;
      if (masked) {
        const uint32_t r = 4 * g + (e & 3);
        if (key + (e >> 2) * 16 + r >= seen || r >= exist[set][e >> 2]) x[e] = -INFINITY;
      }
      top = fmaxf(top, x[e]);
    }
    top = max_halves(max_rows(top));
    // m need not follow the maximum at once: it does when some score is kRise above its last one (of
    // 2^kRise no 32-bit sum takes harm), which spares most steps the rescaling
    if (__any(top > m + (kUp<T> + kRise) || (m == -INFINITY && top > m))) {
      const float m_new = fmaxf(m, top - kUp<T>);
      const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
      m = m_new;
      l_sum.scale(alpha);
#pragma unroll
      for (int j = 0; j < kDims; ++j) o[j] *= alpha;
    }
    const float m_use = m == -INFINITY ? 0.f : m;  // nothing seen so far: all exponentials are 0
    Pack8 p;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      x[e] = __builtin_amdgcn_exp2f(x[e] - m_use);
      put(p, e, x[e], T());
    }
    l_sum.add(sum_of<8>(x));
    if (exist[set][0] + exist[set][1] < 32) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int c = 0; c < kWords; ++c)
          if (4 * g + (e & 3) >= exist[set][e >> 2]) vv[set][e][c] = 0;
    }
    if (looked_at(half)) {
      uint32_t any = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int c = 0; c < kWords; ++c) any |= special_bits<T>(vv[set][e][c]);
      if (__any(any != 0)) {
        special = true;
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int c = 0; c < kWords; ++c) vv[set][e][c] = clear_special<T>(vv[set][e][c]);
      }
    }
#pragma unroll
    for (int c = 0; c < kWords; ++c) {
      Pack8 lo, hi;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        lo.u[e] = __builtin_amdgcn_perm(vv[set][2 * e + 1][c], vv[set][2 * e][c], 0x05040100u);
        hi.u[e] = __builtin_amdgcn_perm(vv[set][2 * e + 1][c], vv[set][2 * e][c], 0x07060302u);
      }
      o[2 * c] = Mfma<T>::run(get(lo, T()), get(p, T()), o[2 * c]);
      o[2 * c + 1] = Mfma<T>::run(get(hi, T()), get(p, T()), o[2 * c + 1]);
    }
  };
  typedef std::integral_constant<int, 0> Even;
  typedef std::integral_constant<int, 1> Odd;
  if (begin < end) load_half(begin, Even());
  for (uint32_t half = begin; half < end; half += 2 * kWaves) {
    do_half(half, Even());
    if (half + kWaves < end) do_half(half + kWaves, Odd());
  }
  if (special) {  // the same halves again: those that were looked at
    for (uint32_t half = begin; half < end; half += kWaves) {
      if (!looked_at(half)) continue;
      const uint32_t key = key_of(half);
      for (uint32_t i = 0; i < 32; ++i) {
        const uint32_t first = key + (i & 16);
        const Keys16 t = keys16(a, page_at(a, own_pages, first, it.own_keys), first, it.own_keys, head);
        if ((i & 15) >= t.n || key + i >= own_seen) continue;
        const uint8_t* const v = t.v + (int64_t)(i & 15) * a.v_place;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          add_special<T, kDims>(v + (g * 4 + r) * kDims * 2, [&](int j, float x) { o[j][r] += x; });
      }
    }
  }

  // the four waves' results, joined through LDS
  float l = l_sum.value();
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (g == 0) {
    lds_m[wave][n] = m;
    lds_l[wave][n] = l;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int j = 0; j < kDims; j += 4) {
      const f32x4 x = {o[j][r], o[j + 1][r], o[j + 2][r], o[j + 3][r]};
      *reinterpret_cast<f32x4*>(&lds_o[wave][n][(g * 4 + r) * kDims + j]) = x;
    }
  __syncthreads();
  constexpr int kQuads = D / 4;
  for (int i = threadIdx.x; i < (int)kFewRows * kQuads; i += kThreads) {
    const uint32_t rr = i / kQuads, c = i % kQuads, in = tile * kFewRows + rr;
    if (in >= rows) continue;
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) top = fmaxf(top, lds_m[v][rr]);
    float sum = 0.f;
    f32x4 acc = (f32x4)0.f;
#pragma unroll
    for (int v = 0; v < kWaves; ++v) {
      const float lv = lds_l[v][rr];
      if (lv == 0.f) continue;  // saw nothing
      const float f = __builtin_amdgcn_exp2f(lds_m[v][rr] - top);
      sum += f * lv;
      acc += f * *reinterpret_cast<const f32x4*>(&lds_o[v][rr][4 * c]);
    }
    if (it.partial) {
      const uint64_t at_row = it.part_first + ((uint64_t)head * it.chunks + chunk) * rows + in;
      *reinterpret_cast<f32x4*>(w.part_o + at_row * D + 4 * c) = acc;
      if (c == 0) {
        w.part_ml[2 * at_row] = top;
        w.part_ml[2 * at_row + 1] = sum;
      }
    } else {
      const uint32_t t = it.token_first + in / a.ratio, h = head * a.ratio + in % a.ratio;
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      scalar y[4];
#pragma unroll
      for (int d = 0; d < 4; ++d) y[d] = (scalar)(acc[d] * inv);
      const uint64_t to = (uint64_t)t * a.q_heads + h;
      *reinterpret_cast<uint64_t*>(a.out + (to * D + 4 * c) * 2) = *reinterpret_cast<const uint64_t*>(y);
      if (c == 0 && a.lse) a.lse[to] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
    }
  }
}

// 128 rows, 32 a wave, over keys that the workgroup stages in LDS: a sub-step's keys are loaded
// into registers two sub-steps ahead, and stored one ahead. A SIMD has one wave of each of two
// workgroups: as these share no barrier, the products of one go on under the other's softmax.
// 8,192 tokens of 32 heads of 128: 630 to 680 us from box to box, 810 to 870 TFLOP/s, where a library
// product of 8,192 cubed reaches 1,150 to 1,280. No unit is the limit by itself: of a step's 1.3 us
// its products take 0.4, the exponentials with the rest of the softmax 0.5, the LDS 0.5, as counted
// from the instructions at 2.4 GHz. With heads of 256, of one workgroup a CU and a barrier every 32
// keys, 4,096 tokens of 16 heads on 4 take 284 us, 480 TFLOP/s (heads of 128: 118 us, 580).
//
// Products are v_mfma_f32_32x32x16 in the same orientation: S^T = K Q^T, O^T = V^T P^T, a lane
// holding one row's scores with keys 8 i + 4 h .. + 3 (h = lane / 32), which again are P's operand
// as they are when V's brings keys {4h..} and {8 + 4h..} of each 16. V's operand, 8 keys of one
// dim, comes from rows in LDS through the transposing ds_read_b64_tr_b16: 16 lanes read 4 keys of
// 16 dims, and lane i gets dim i of all 4. Rows in LDS are swizzled so that the lanes of one read
// fall into different banks: 16-byte pieces of K by the row, 32-byte pieces of V by the row's
// place among the 4.
template <int D>
struct Staged {
  static constexpr int kKeys = D == 256 ? 32 : 64;      // keys of a sub-step
  static constexpr int kSubs = kStep / kKeys;           // sub-steps of a step
  static constexpr int kRow = 2 * D;                    // bytes of a row
  static constexpr int kPieces = kRow / 16;             // 16-byte pieces of a row
  static constexpr int kRows = kKeys / kWaves;          // rows that a wave stages
  static constexpr int kLoads = kRows * kPieces / 64;   // 16-byte loads of a lane for them
  static constexpr int kTile = kKeys * kRow;            // bytes of K or V
  static constexpr int kBytes = 4 * kTile + 2 * kWaves; // two of each, and flags
  static __device__ uint32_t k_at(uint32_t row, uint32_t piece) {
    return row * kRow + ((piece ^ (D == 64 ? (row >> 1) & 7 : row & 15)) << 4);
  }
  static __device__ uint32_t v_swizzle(uint32_t row) { return D == 64 ? ((row >> 1) & 1) << 1 : (row & 3) << 1; }
  static __device__ uint32_t v_at(uint32_t row, uint32_t piece) {
    return row * kRow + (((piece >> 1) ^ v_swizzle(row)) << 5) + ((piece & 1) << 4);
  }
};

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

template <class T> struct Mfma32;
template <> struct Mfma32<Fp16> {
  static __device__ f32x16 run(f16x8 a, f16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};
template <> struct Mfma32<Bf16> {
  static __device__ f32x16 run(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};

__device__ inline u32x2v read_transposed(const char* p) {
  union {
    s16x4 s;
    u32x2v u;
  } x;
  x.s = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(__attribute__((address_space(3))) void*)const_cast<char*>(p));
  return x.u;
}

template <class T, int D>
__device__ __forceinline__ void attend_tile(const AttendArgs& a, const Unit& unit, char* lds) {
  typedef typename T::scalar scalar;
  typedef Staged<D> St;
  constexpr int kKTiles = St::kKeys / 32, kQ = D / 16, kO = D / 32;
  char* const lds_k = lds;
  char* const lds_v = lds + 2 * St::kTile;
  uint8_t* const lds_flags = reinterpret_cast<uint8_t*>(lds + 4 * St::kTile);
  // of a wave's staged rows: how many exist, in a byte, 0x80 added where values were cleared
  constexpr uint32_t kWhole = St::kRows * 0x01010101u, kCleared = 0x80808080u;
  const Item& it = unit.it;
  const uint32_t head = unit.head, rows = it.tokens * a.ratio;
  const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const uint32_t n = lane & 31, h = lane >> 5;
  const uint32_t wave_row = unit.tile * kTileRows + 32 * wave;
  const uint32_t row = wave_row + n;
  const bool row_live = row < rows;
  const uint32_t token = it.token_first + (row_live ? row / a.ratio : 0);
  const uint32_t q_head = head * a.ratio + (row_live ? row % a.ratio : 0);

  // keys of the sequence's own that the lane's row sees, the fewest and most of the wave's rows,
  // and of the workgroup's
  const int64_t behind = (int64_t)it.own_keys - it.tokens + 1;
  auto seen_by = [&](uint32_t r) {
    if (r >= rows) r = rows - 1;
    const int64_t x = behind + r / a.ratio;
    return x < 0 ? 0u : (uint32_t)x;
  };
  const uint32_t own_seen = seen_by(row), own_least = uniform(seen_by(wave_row));
  const uint32_t own_wave_most = uniform(wave_row < rows ? seen_by(wave_row + 31) : 0);
  const uint32_t own_group_least = uniform(seen_by(unit.tile * kTileRows));
  const uint32_t own_most = uniform(seen_by(unit.tile * kTileRows + kTileRows - 1));

  // Scores are scaled after the product, and masked ones are minus infinity before it: a scale below
  // zero is taken from the queries' signs, so that the largest score is the largest product's, and
  // one of zero is taken as queries of zero, NaN where the query is infinite or NaN.
  const float scale = a.scale_log2 == 0.f ? 1.f : fabsf(a.scale_log2);
  Pack8 q[kQ];
#pragma unroll
  for (int i = 0; i < kQ; ++i) {
    q[i].u = (u32x4v)0u;
    if (row_live)
      q[i].u = *reinterpret_cast<const u32x4v*>(a.q + (int64_t)token * a.q_token + (int64_t)q_head * a.q_head +
                                                (i * 16 + h * 8) * 2);
  }

  const int32_t* const prefix_pages = a.prefix_pages + (uint64_t)it.prefix_row * a.prefix_width;
  const int32_t* const own_pages = a.own_pages + (uint64_t)it.own_row * a.own_width;
  const uint32_t prefix_subs = St::kSubs * steps_of(it.prefix_keys);
  const uint32_t all_subs = prefix_subs + (own_most + St::kKeys - 1) / St::kKeys;
  uint32_t end = St::kSubs * (unit.chunk + 1) * it.per;
  if (end > all_subs) end = all_subs;
  const uint32_t first = St::kSubs * unit.chunk * it.per;
  // after wave_end the wave's rows see nothing (rows that do not exist, from the start): it only stages
  uint32_t wave_end = wave_row < rows ? prefix_subs + (own_wave_most + St::kKeys - 1) / St::kKeys : first;
  if (wave_end > end) wave_end = end;

  // of the wave's rows of a sub-step the first key, and all keys there are; its page for the 64
  // sub-steps from page_sub on, one a lane
  auto keys_of = [&](uint32_t s) { return s < prefix_subs ? it.prefix_keys : it.own_keys; };
  auto key_of = [&](uint32_t s) {
    return (s < prefix_subs ? s : s - prefix_subs) * St::kKeys + wave * St::kRows;
  };
  auto pages_from = [&](uint32_t s) {
    s += lane;
    if (s >= end) return kNoPage;
    return page_at(a, s < prefix_subs ? prefix_pages : own_pages, key_of(s), keys_of(s));
  };
  uint32_t page_sub = first, pages = pages_from(first);

  // Those rows, from memory to registers and from there to LDS. All of them are loaded, whether keys
  // or not: they lie in one page, and in the cache's first where there is no page (without keys
  // there are no sub-steps, without pages no keys). Keys that are none are masked, and the values
  // in their place set to 0.
  constexpr uint32_t kLoadRows = 64 / St::kPieces;  // rows of one load
  const uint32_t piece = lane % St::kPieces, load_row = lane / St::kPieces;
  const uint32_t k_off = load_row * (uint32_t)a.k_place + piece * 16;
  const uint32_t v_off = load_row * (uint32_t)a.v_place + piece * 16;
  u32x4v stage_k[St::kLoads], stage_v[St::kLoads];
  uint32_t stage_flags = 0;
  auto stage_load = [&](uint32_t s) {
    if (s - page_sub >= 64) {
      page_sub = s;
      pages = pages_from(s);
    }
    const uint32_t page = (uint32_t)__builtin_amdgcn_readlane((int)pages, (int)(s - page_sub));
    const Keys16 t = keys16(a, page, key_of(s), keys_of(s), head);
    stage_flags = t.n < (uint32_t)St::kRows ? t.n : (uint32_t)St::kRows;
#pragma unroll
    for (int i = 0; i < St::kLoads; ++i) stage_k[i] = load_at<u32x4v>(t.k + i * kLoadRows * a.k_place, k_off);
#pragma unroll
    for (int i = 0; i < St::kLoads; ++i) stage_v[i] = load_at<u32x4v>(t.v + i * kLoadRows * a.v_place, v_off);
  };
  auto stage_tidy = [&](uint32_t s) {
    if (stage_flags < (uint32_t)St::kRows) {
#pragma unroll
      for (int i = 0; i < St::kLoads; ++i)
        if (i * kLoadRows + load_row >= stage_flags) stage_v[i] = (u32x4v)0u;
    }
    if (s >= prefix_subs && (s - prefix_subs + 1) * St::kKeys > own_group_least) {
      uint32_t any = 0;
#pragma unroll
      for (int i = 0; i < St::kLoads; ++i)
#pragma unroll
        for (int c = 0; c < 4; ++c) any |= special_bits<T>(stage_v[i][c]);
      if (__any(any != 0)) {
        stage_flags |= 0x80;
#pragma unroll
        for (int i = 0; i < St::kLoads; ++i)
#pragma unroll
          for (int c = 0; c < 4; ++c) stage_v[i][c] = clear_special<T>(stage_v[i][c]);
      }
    }
  };
  auto stage_store = [&](uint32_t s) {
    const uint32_t buf = (s - first) & 1;
#pragma unroll
    for (int i = 0; i < St::kLoads; ++i) {
      const uint32_t r = wave * St::kRows + i * kLoadRows + load_row;
      *reinterpret_cast<u32x4v*>(lds_k + buf * St::kTile + St::k_at(r, piece)) = stage_k[i];
      *reinterpret_cast<u32x4v*>(lds_v + buf * St::kTile + St::v_at(r, piece)) = stage_v[i];
    }
    if (lane == 0) lds_flags[buf * kWaves + wave] = (uint8_t)stage_flags;
  };

  bool special = false;
  float m = -INFINITY;  // of the products, not yet scaled, without kUp
  Sum l_sum;
  f32x16 o[kO];
#pragma unroll
  for (int i = 0; i < kO; ++i) o[i] = (f32x16)0.f;

  // where the lane reads: K rows and pieces, V quads of keys and dims
  const uint32_t k_lane = St::k_at(n, h);
  const uint32_t v_row = 4 * h + ((lane & 15) >> 2);
  const uint32_t v_lane = v_row * St::kRow + ((((lane >> 4) & 1) ^ St::v_swizzle(v_row)) << 5) + (lane & 3) * 8;

  if (first < end) {
    stage_load(first);
    stage_tidy(first);
    stage_store(first);
    if (first + 1 < end) stage_load(first + 1);
  }
  // the queries as the scale wants them: here, where they have arrived
  const uint32_t flip = a.scale_log2 < 0.f ? 0x80008000u : 0u;
#pragma unroll
  for (int i = 0; i < kQ; ++i) q[i].u ^= flip;
  if (a.scale_log2 == 0.f) {
#pragma unroll
    for (int i = 0; i < kQ; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) q[i].u[c] = (special_bits<T>(q[i].u[c]) >> 15) * 0x7fffu;
  }
  // One barrier a sub-step: what it stores one ahead is complete at the next one's, and goes to the
  // buffer that all waves were done with at its own.
  for (uint32_t sub = first; sub < end; ++sub) {
    const uint32_t buf = (sub - first) & 1;
    __syncthreads();
    if (sub + 1 < end) {
      stage_tidy(sub + 1);
      stage_store(sub + 1);
    }
    if (sub + 2 < end) stage_load(sub + 2);
    if (sub < wave_end) {
      const bool shared = sub < prefix_subs;
      const uint32_t key = (shared ? sub : sub - prefix_subs) * St::kKeys;
      const char* const kb = lds_k + buf * St::kTile;
      const char* const vb = lds_v + buf * St::kTile;
      const uint32_t flags = uniform(*reinterpret_cast<const uint32_t*>(lds_flags + buf * kWaves));
      special |= (flags & kCleared) != 0;
      f32x16 s[kKTiles];
#pragma unroll
      for (int t = 0; t < kKTiles; ++t) {
        s[t] = (f32x16)0.f;
#pragma unroll
        for (int i = 0; i < kQ; ++i) {
          Pack8 k;
          k.u = *reinterpret_cast<const u32x4v*>(kb + t * 32 * St::kRow + (k_lane ^ (i << 5)));
          s[t] = Mfma32<T>::run(get(k, T()), get(q[i], T()), s[t]);
        }
      }
      const bool all_exist = (flags & ~kCleared) == kWhole;
      if (!all_exist || (!shared && key + St::kKeys > own_least)) {
        const uint32_t seen = shared ? it.prefix_keys : own_seen;
#pragma unroll
        for (int t = 0; t < kKTiles; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int quad = 32 * t + 8 * (r / 4);  // and 4 h on
            const uint32_t in = quad % St::kRows + r % 4 + 4 * h, w = quad / St::kRows;  // in wave w's rows
            const uint32_t exist = (flags >> (8 * w)) & 0x7f;
            if (key + w * St::kRows + in >= seen || in >= exist) s[t][r] = -INFINITY;
          }
      }
      float top = s[0][0];
#pragma unroll
      for (int t = 0; t < kKTiles; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
      top = max_halves(top);
      // m need not be the maximum itself: it follows once some score is kRise above it (as above)
      if (__any((top - m) * scale > kRise || (m == -INFINITY && top > m))) {
        const float m_new = fmaxf(m, top);
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - m_new) * scale);
        m = m_new;
        l_sum.scale(alpha);
#pragma unroll
        for (int i = 0; i < kO; ++i) o[i] *= alpha;
      }
      const float bias = m == -INFINITY ? 0.f : kUp<T> - m * scale;  // nothing seen so far: all exponentials are 0
      Pack8 p[kKTiles * 2];
      float step = 0.f;
#pragma unroll
      for (int t = 0; t < kKTiles; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float y = __builtin_amdgcn_exp2f(fmaf(s[t][r], scale, bias));
          step += y;
          put(p[2 * t + r / 8], r % 8, y, T());
        }
      l_sum.add(step);
#pragma unroll
      for (int kk = 0; kk < 2 * kKTiles; ++kk)
#pragma unroll
        for (int i = 0; i < kO; ++i) {
          Pack8 v;
          const u32x2v x = read_transposed(vb + kk * 16 * St::kRow + (v_lane ^ (i << 6)));
          const u32x2v y = read_transposed(vb + (kk * 16 + 8) * St::kRow + (v_lane ^ (i << 6)));
          v.u = (u32x4v){x[0], x[1], y[0], y[1]};
          o[i] = Mfma32<T>::run(get(v, T()), get(p[kk], T()), o[i]);
        }
    }
  }

  const float l = sum_halves(l_sum.value());
  if (!row_live) return;
  if (special) {
    uint32_t key = own_group_least & ~(St::kKeys - 1u);  // the first sub-step that was looked at
    if (first > prefix_subs && (first - prefix_subs) * St::kKeys > key) key = (first - prefix_subs) * St::kKeys;
    const uint32_t to = (end - prefix_subs) * St::kKeys;
    for (; key < to && key < own_seen; ++key) {
      const Keys16 t = keys16(a, page_at(a, own_pages, key & ~15u, it.own_keys), key & ~15u, it.own_keys, head);
      if ((key & 15) >= t.n) continue;
      const uint8_t* const v = t.v + (int64_t)(key & 15) * a.v_place + 8 * h;
#pragma unroll
      for (int i = 0; i < kO; ++i)
#pragma unroll
        for (int r = 0; r < 16; r += 4)
          add_special<T, 4>(v + (32 * i + 2 * r) * 2, [&](int c, float x) { o[i][r + c] += x; });
    }
  }
  const float top = m == -INFINITY ? -INFINITY : m * scale - kUp<T>;
  if (it.partial) {
    const uint64_t at_row = it.part_first + ((uint64_t)head * it.chunks + unit.chunk) * rows + row;
    float* const to = a.ws.part_o + at_row * D + 4 * h;
#pragma unroll
    for (int i = 0; i < kO; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        *reinterpret_cast<f32x4*>(to + 32 * i + 2 * r) = (f32x4){o[i][r], o[i][r + 1], o[i][r + 2], o[i][r + 3]};
    if (h == 0) {
      a.ws.part_ml[2 * at_row] = top;
      a.ws.part_ml[2 * at_row + 1] = l;
    }
  } else {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const uint64_t to = (uint64_t)token * a.q_heads + q_head;
    scalar* const out = reinterpret_cast<scalar*>(a.out) + to * D + 4 * h;
#pragma unroll
    for (int i = 0; i < kO; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        scalar y[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] = (scalar)(o[i][r + c] * inv);
        *reinterpret_cast<uint64_t*>(out + 32 * i + 2 * r) = *reinterpret_cast<const uint64_t*>(y);
      }
    if (h == 0 && a.lse) a.lse[to] = l == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * kLn2;
  }
}

template <int D>
constexpr int lds_bytes() {
  constexpr int few = kWaves * kFewRows * (D + 4 + 2) * 4, tile = Staged<D>::kBytes;
  return few > tile ? few : tile;
}

template <class T, int D>
__global__ __launch_bounds__(kThreads, D == 256 ? 1 : 2) void attend_kernel(AttendArgs a) {
  __shared__ __attribute__((aligned(16))) char lds[lds_bytes<D>()];
  const Ws& w = a.ws;
  const uint32_t n_items = a.n_groups + a.n_seq, lane = threadIdx.x & 63;
  // units of full tiles come first
  uint32_t tiles, fews;
  WavePlan plan;
  const bool in_wave = n_items <= kWaveItems;
  if (in_wave) {
    plan = plan_in_wave(a);
    if (blockIdx.x == 0 && threadIdx.x < 64) write_plan(a, plan);
    tiles = plan.tiles;
    fews = plan.fews;
  } else {
    tiles = w.head->tiles;
    fews = w.head->fews;
  }
  tiles = uniform(tiles);
  fews = uniform(fews);
  if (blockIdx.x >= tiles + fews) return;
  const bool few = blockIdx.x >= tiles;
  uint32_t u = few ? blockIdx.x - tiles : blockIdx.x;
  Unit unit;
  if (in_wave) {
    const uint64_t le = __ballot(lane < n_items && (few ? plan.it.few_first : plan.it.tile_first) <= u);
    unit.it = item_of_lane(plan.it, 63 - __clzll((long long)le));
  } else {
    unit.it = w.items[uniform(wave_search<uint32_t>(few ? w.few_first : w.tile_first, n_items, u))];
  }
  u -= few ? unit.it.few_first : unit.it.tile_first;
  unit.head = u % a.kv_heads;
  u /= a.kv_heads;
  unit.chunk = u % unit.it.chunks;
  // a prompt's last rows see the most keys: they come first
  unit.tile = tiles_of(unit.it.tokens * a.ratio) - 1 - u / unit.it.chunks;
  unit.it = item_of_lane(unit.it, 0);
  unit.head = uniform(unit.head);
  unit.chunk = uniform(unit.chunk);
  unit.tile = uniform(unit.tile);
  if (few) attend_few<T, D>(a, unit, lds);
  else attend_tile<T, D>(a, unit, lds);
}

// D/4 lanes take a piece of a row, 4 dims each. Where there are many rows they join all of its
// pieces, 64 / (D/4) rows a wave; with few rows (kWide) a workgroup's lanes share the pieces of
// one. Four pieces are in flight at a time. Bound by reading the pieces, or with few by the time
// of half a dozen loads that wait for each other: 4 to 5 us, 7 for 2,048 rows of some ten pieces, 2
// where no row has pieces.
// Rows that no piece covers are set to nothing seen.
template <class T, int D, bool kWide>
__global__ __launch_bounds__(kThreads) void join_kernel(AttendArgs a) {
  typedef typename T::scalar scalar;
  constexpr uint32_t kLanes = D / 4, kTeams = kThreads / kLanes;
  constexpr uint32_t kRows = kWide ? 1 : kTeams, kStride = kWide ? kTeams : 1;
  __shared__ __attribute__((aligned(16))) float lds_o[kWide ? kTeams : 1][D];
  __shared__ float lds_m[kTeams], lds_l[kTeams];
  const Ws& w = a.ws;
  // asked for together: each comes from memory, as another kernel has just written it
  uint32_t joins = 1;
  int32_t t0 = 0, t1 = 0;
  if (a.n_seq) {
    joins = w.head->joins;
    t0 = w.q_first[0];
    t1 = w.q_first[a.n_seq];
  }
  asm volatile("" : "+v"(joins), "+v"(t0), "+v"(t1));
  if (!joins) return;  // attend_kernel wrote every row
  const uint32_t team = threadIdx.x / kLanes, dim = threadIdx.x % kLanes * 4;
  const uint32_t all = a.n_tokens * a.q_heads;
  // the rows of a workgroup are side by side: of few tokens, and the first one's sequence is found by all
  for (uint32_t r0 = blockIdx.x * kRows; r0 < all; r0 += gridDim.x * kRows) {
    const uint32_t token0 = r0 / a.q_heads;
    uint32_t s = 0;
    if ((int32_t)token0 >= t0 && (int32_t)token0 < t1) s = wave_search<int32_t>(w.q_first, a.n_seq, (int32_t)token0);
    const uint32_t r = r0 + (kWide ? 0 : team);
    if (r >= all) continue;
    const uint32_t token = r / a.q_heads, h = r - token * a.q_heads;
    const uint32_t head = h / a.ratio;
    uint32_t first[2] = {0, 0}, count[2] = {0, 0}, step[2] = {0, 0};  // the group's pieces, the sequence's
    if ((int32_t)token >= t0 && (int32_t)token < t1) {
      while (w.q_first[s + 1] <= (int32_t)token) ++s;
      const Item& own = w.items[a.n_groups + s];
      const uint32_t chunks = own.chunks, partial = own.partial;
      const int32_t gr = a.n_groups ? w.seq_group[s] : -1;
      if (!partial && chunks) continue;  // written already
      if (partial) {
        const uint32_t rows = own.tokens * a.ratio;
        first[1] = own.part_first + head * chunks * rows + (token - own.token_first) * a.ratio + h % a.ratio;
        count[1] = chunks;
        step[1] = rows;
        if (gr >= 0) {
          const Item& pre = w.items[gr];
          const uint32_t all_rows = pre.tokens * a.ratio;
          first[0] = pre.part_first + head * pre.chunks * all_rows + (token - pre.token_first) * a.ratio + h % a.ratio;
          count[0] = pre.chunks;
          step[0] = all_rows;
        }
      }
    }
    const uint32_t pieces = count[0] + count[1];
    float m = -INFINITY, l = 0.f;
    f32x4 acc = (f32x4)0.f;
    for (uint32_t p0 = kWide ? team : 0; p0 < pieces; p0 += 4 * kStride) {
      float pm[4], pl[4];
      f32x4 x[4];
#pragma unroll
      for (uint32_t u = 0; u < 4; ++u) {
        const uint32_t p = p0 + u * kStride;
        pm[u] = -INFINITY;
        pl[u] = 0.f;
        x[u] = (f32x4)0.f;
        if (p < pieces) {
          const uint64_t at = p < count[0] ? first[0] + p * step[0] : first[1] + (p - count[0]) * step[1];
          pm[u] = w.part_ml[2 * at];
          pl[u] = w.part_ml[2 * at + 1];
          x[u] = *reinterpret_cast<const f32x4*>(w.part_o + at * D + dim);
        }
      }
      float m_new = m;
#pragma unroll
      for (uint32_t u = 0; u < 4; ++u) m_new = fmaxf(m_new, pm[u]);
      const float m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(m - m_use);
      m = m_new;
      l *= alpha;
      acc *= alpha;
#pragma unroll
      for (uint32_t u = 0; u < 4; ++u) {
        if (pl[u] == 0.f) continue;  // saw nothing
        const float f = __builtin_amdgcn_exp2f(pm[u] - m_use);
        l += f * pl[u];
        acc += f * x[u];
      }
    }
    if constexpr (kWide) {
      if (dim == 0) {
        lds_m[team] = m;
        lds_l[team] = l;
      }
      *reinterpret_cast<f32x4*>(&lds_o[team][dim]) = acc;
      __syncthreads();
      if (team != 0) return;  // one row a workgroup
      m = lds_m[0];
#pragma unroll
      for (uint32_t i = 1; i < kTeams; ++i) m = fmaxf(m, lds_m[i]);
      l = 0.f;
      acc = (f32x4)0.f;
#pragma unroll
      for (uint32_t i = 0; i < kTeams; ++i) {
        if (lds_l[i] == 0.f) continue;
        const float f = __builtin_amdgcn_exp2f(lds_m[i] - m);
        l += f * lds_l[i];
        acc += f * *reinterpret_cast<const f32x4*>(&lds_o[i][dim]);
      }
    }
    const bool none = l == 0.f;
    const float inv = none ? 0.f : 1.f / l;
    scalar y[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) y[d] = (scalar)(acc[d] * inv);
    *reinterpret_cast<uint64_t*>(a.out + ((uint64_t)r * D + dim) * 2) = *reinterpret_cast<const uint64_t*>(y);
    if (a.lse && dim == 0) a.lse[r] = none ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
  }
}

// Sets the error text with the call's name; *shape and *args as the kernels take them.
gleam_status validate_attention(const gleam_kv_pages* kv, const gleam_prefix_batch* b, PlanShape* shape) {
  const char* const who = "gleam_prefix_attention";
  gleam_status st = validate_kv(kv, who);
  if (st != GLEAM_OK) return st;
  if (!b) {
    set_error("%s: null batch", who);
    return GLEAM_E_INVALID;
  }
  if (b->q_heads == 0 || b->q_heads % kv->kv_heads != 0 || b->q_heads > 65535) {
    set_error("%s: q_heads must be a multiple of kv_heads, up to 65535", who);
    return GLEAM_E_INVALID;
  }
  // places of 16 keys are reached by 32-bit offsets
  if (kv->k_stride[1] >= 1 << 26 || kv->v_stride[1] >= 1 << 26) {
    set_error("%s: places of a page 2^26 elements apart or more", who);
    return GLEAM_E_UNSUPPORTED;
  }
  if (b->n_tokens > (uint64_t)INT32_MAX / b->q_heads) {
    set_error("%s: n_tokens * q_heads of 2^31 or more", who);
    return GLEAM_E_UNSUPPORTED;
  }
  if (b->n_seq > kMostSeq || b->n_groups > kMostSeq) {
    set_error("%s: more than 2^20 sequences or groups", who);
    return GLEAM_E_UNSUPPORTED;
  }
  if (b->own_width > (uint64_t)INT32_MAX / kv->page_tokens || b->prefix_width > (uint64_t)INT32_MAX / kv->page_tokens) {
    set_error("%s: a table row of 2^31 keys or more", who);
    return GLEAM_E_INVALID;
  }
  shape->n_tokens = b->n_tokens;
  shape->n_seq = b->n_seq;
  shape->n_groups = b->n_groups;
  shape->kv_heads = kv->kv_heads;
  shape->ratio = b->q_heads / kv->kv_heads;
  shape->target = kUnits;
  shape->head_dim = kv->head_dim;
  const uint64_t most = steps_of((uint32_t)(b->own_width * kv->page_tokens)) +
                        (uint64_t)steps_of((uint32_t)(b->prefix_width * kv->page_tokens));
  shape->most_steps = (uint32_t)most;
  if (most_units_any_width(*shape) > max_workgroups(kThreads) || most_partials(*shape) > UINT32_MAX) {
    set_error("%s: more work than one launch holds", who);
    return GLEAM_E_UNSUPPORTED;
  }
  return GLEAM_OK;
}

template <class T, int D>
gleam_status launch_all(const AttendArgs& a, uint32_t units, hipStream_t stream) {
  gleam_status st;
  const uint32_t items = a.n_groups + a.n_seq;
  if (items > kWaveItems && a.n_seq > 0) {
    // as few threads as hold the offsets: a barrier of 16 waves takes longer than one of 3
    const uint32_t threads = items < kPlanThreads ? (items + 64) / 64 * 64 : kPlanThreads;
    hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(threads), 0, stream, a);
    if ((st = launch_status("plan_kernel")) != GLEAM_OK) return st;
  }
  if (units > 0) {
    hipLaunchKernelGGL((attend_kernel<T, D>), dim3(units), dim3(kThreads), 0, stream, a);
    if ((st = launch_status("attend_kernel")) != GLEAM_OK) return st;
  }
  const uint32_t rows = a.n_tokens * a.q_heads;
  if (rows <= kWideJoin) {
    hipLaunchKernelGGL((join_kernel<T, D, true>), dim3(rows), dim3(kThreads), 0, stream, a);
  } else {
    constexpr uint32_t per = kThreads / (D / 4);
    const uint32_t groups = (rows + per - 1) / per;
    hipLaunchKernelGGL((join_kernel<T, D, false>), dim3(groups < kMostJoins ? groups : kMostJoins), dim3(kThreads), 0,
                       stream, a);
  }
  return launch_status("join_kernel");
}

}  // namespace

hipError_t preload_prefix_attention() {
  hipFuncAttributes attr;
  return hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&plan_kernel));
}

}  // namespace gleam

extern "C" size_t gleam_prefix_attention_ws_bytes(const gleam_kv_pages* kv, const gleam_prefix_batch* b) {
  using namespace gleam;
  clear_error();
  PlanShape s{};
  if (validate_attention(kv, b, &s) != GLEAM_OK) return 0;
  return ws_at(nullptr, s, kv->head_dim).bytes;
}

extern "C" gleam_status gleam_prefix_attention(const gleam_kv_pages* kv, const gleam_prefix_batch* b, void* d_out,
                                               float* d_lse, void* d_ws, size_t ws_bytes, void* stream) {
  using namespace gleam;
  clear_error();
  const char* const who = "gleam_prefix_attention";
  PlanShape shape{};
  gleam_status st = validate_attention(kv, b, &shape);
  if (st != GLEAM_OK) return st;
  if (b->n_tokens == 0) return GLEAM_OK;
  if ((st = validate_heads(b->d_q, b->q_stride, "q", who)) != GLEAM_OK) return st;
  const int64_t whole[2] = {0, 0};
  if ((st = validate_heads(d_out, whole, "out", who)) != GLEAM_OK) return st;
  if (b->n_seq > 0 && (!b->d_q_first || !b->d_own_len || (b->own_width > 0 && !b->d_own_pages))) {
    set_error("%s: null q_first, own_len or own_pages", who);
    return GLEAM_E_INVALID;
  }
  if (b->n_groups > 0 && (!b->d_group_first || !b->d_prefix_len || (b->prefix_width > 0 && !b->d_prefix_pages))) {
    set_error("%s: groups need group_first, prefix_len and prefix_pages", who);
    return GLEAM_E_INVALID;
  }
  if (!d_ws || !aligned256(d_ws)) {
    set_error("%s: workspace must be non-null and 256-byte aligned", who);
    return GLEAM_E_INVALID;
  }
  AttendArgs a{};
  a.ws = ws_at(static_cast<uint8_t*>(d_ws), shape, kv->head_dim);
  if (ws_bytes < a.ws.bytes) {
    set_error("%s: workspace of %zu bytes, %zu needed", who, ws_bytes, a.ws.bytes);
    return GLEAM_E_WORKSPACE;
  }
  a.q = static_cast<const uint8_t*>(b->d_q);
  a.q_token = 2 * b->q_stride[0];
  a.q_head = 2 * b->q_stride[1];
  a.k = static_cast<const uint8_t*>(kv->d_k);
  a.v = static_cast<const uint8_t*>(kv->d_v);
  a.k_page = 2 * kv->k_stride[0];
  a.k_place = 2 * kv->k_stride[1];
  a.k_head = 2 * kv->k_stride[2];
  a.v_page = 2 * kv->v_stride[0];
  a.v_place = 2 * kv->v_stride[1];
  a.v_head = 2 * kv->v_stride[2];
  a.q_first = b->d_q_first;
  a.own_pages = b->d_own_pages;
  a.own_len = b->d_own_len;
  a.group_first = b->d_group_first;
  a.prefix_pages = b->d_prefix_pages;
  a.prefix_len = b->d_prefix_len;
  a.n_tokens = (uint32_t)b->n_tokens;
  a.n_seq = (uint32_t)b->n_seq;
  a.n_groups = b->n_seq ? (uint32_t)b->n_groups : 0;
  a.own_width = (uint32_t)b->own_width;
  a.prefix_width = (uint32_t)b->prefix_width;
  a.q_heads = b->q_heads;
  a.kv_heads = kv->kv_heads;
  a.ratio = shape.ratio;
  a.page_log2 = (uint32_t)log2_exact(kv->page_tokens);
  a.n_pages = (uint32_t)kv->n_pages;
  a.target = shape.target;
  a.head_dim = kv->head_dim;
  a.scale_log2 = b->scale * kLog2e;
  a.out = static_cast<uint8_t*>(d_out);
  a.lse = d_lse;
  // no sequences: join_kernel clears all rows; otherwise the first workgroup may leave the plan
  uint32_t units = b->n_seq ? (uint32_t)most_units(shape) : 0;
  if (b->n_seq && units == 0) units = 1;
  hipStream_t s = (hipStream_t)stream;
  if (kv->dtype == GLEAM_FP16) {
    return kv->head_dim == 64    ? launch_all<Fp16, 64>(a, units, s)
           : kv->head_dim == 128 ? launch_all<Fp16, 128>(a, units, s)
                                 : launch_all<Fp16, 256>(a, units, s);
  }
  return kv->head_dim == 64    ? launch_all<Bf16, 64>(a, units, s)
         : kv->head_dim == 128 ? launch_all<Bf16, 128>(a, units, s)
                               : launch_all<Bf16, 256>(a, units, s);
}
