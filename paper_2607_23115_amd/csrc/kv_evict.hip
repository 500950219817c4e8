// Keeping a paged cache within a budget: of each sequence's keys, those of a head that gathered the least
// attention make room. Each key head chooses for itself, all keep as many, so the page table and the
// length hold for all heads.
//
// The order of a sequence's keys means nothing to attention (positions are rotated into the keys, and the
// next tokens' keys come behind), so nothing is shifted: kept keys that lie behind the budget move into the
// places within it that come free, the i-th such key into the i-th such place. A sequence a few tokens over
// its budget moves a few keys, not all of them, and no place that is read is written.
//
// A workgroup chooses for each sequence and head: weights become integers of the same order, that of the last
// key kept is found in four rounds of counting eight bits, then two running counts in the keys' order: of the
// keys of just that weight, to keep the first ones (unless all are kept), and of places that come free and keys
// that move. Where there are many sequences and heads, the workgroup also copies its pairs; with few,
// move_kernel does, over all CUs. A chain of short steps that wait for each other; loops are kept rolled, as
// each instruction runs a few times only and a CU has to fetch it first (with a thread's keys in registers and
// loops unrolled 16 times 64 sequences took 20 to 23 us). 64 sequences of 1,990 to 2,112 keys cut to 2,048, 8 heads
// of 128, take 17 us: 7 until the weights are there, 4 for the rounds, 2 to 3 for the counts, 3 to 4 for the copies;
// 8 prompts of 5,000 to 30,000 keys cut to 1,024 29 us for the choice, on 64 CUs, and 17 for 57 MB of copies.

#include "kv_device.h"
#include "launch_shape.h"

namespace gleam {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
// Keys of a thread, in LDS: for tables of up to 4,096 keys, and for wider ones. Longer sequences than those
// hold read their weights again for each count.
constexpr int kNarrowKeys = 4, kWideKeys = 32;
// Counts of a round, in four copies: weights have few exponents, and lanes that add to the same count wait.
constexpr uint32_t kBins = 256, kCopies = 4, kRound = kBins * kCopies;
constexpr int kMoveThreads = 256;
constexpr uint32_t kMoveGroups = 2048;  // of move_kernel
constexpr uint64_t kMostPairs = 1ull << 36;
// From this many sequences times heads on a narrow table's workgroups copy their pairs themselves: with 256 (32
// sequences, 2,400 keys cut to 2,048) 34 us, by move_kernel 41; with 128 (16 of 4,000 keys to 2,048) 66 and 53.
constexpr uint32_t kManyPairs = 256;

struct EvictArgs {
  uint8_t* base[2];  // keys, values
  int64_t page[2], place[2], head[2];  // bytes
  const int32_t* own_pages;
  const int32_t* own_len;
  const float* weights;
  const int32_t* born;
  const int32_t* total;
  float* weights_out;
  int32_t* born_out;
  int32_t* len_out;
  uint32_t* moves;  // [n_seq][kv_heads]
  uint2* pairs;     // [n_seq][kv_heads][most]: the place a key leaves and the one that it goes to
  uint32_t most;
  uint32_t copies;  // select_kernel copies the pairs
  uint32_t n_seq, own_width, page_log2, n_pages, kv_heads, keep, sinks, recent;
};

__device__ inline uint32_t keys_of(const EvictArgs& a, uint32_t s) {
  return a.n_pages ? (uint32_t)clamp_to(a.own_len[s], (int32_t)(a.own_width << a.page_log2)) : 0;
}

// Where key i's weight and birth are; ~0 in a page that the cache does not have.
__device__ inline uint64_t tracked_at(const EvictArgs& a, const int32_t* pages, uint32_t head, uint32_t i) {
  const uint32_t page = (uint32_t)pages[i >> a.page_log2];
  if (page >= a.n_pages) return ~0ull;
  return ((uint64_t)page * a.kv_heads + head) << a.page_log2 | (i & ((1u << a.page_log2) - 1));
}

// A larger number for a larger weight: 1 for NaN (0 is a key's in a page that is none), -0 as 0.
__device__ inline uint32_t order_of(float w) {
  const uint32_t b = __float_as_uint(w + 0.f);
  return w != w ? 1 : b ^ ((b >> 31) ? ~0u : 0x80000000u);
}

// What a key counts for: ~0 for one that is kept whatever its weight.
__device__ inline uint32_t rank_of(const EvictArgs& a, float w, int32_t born, int64_t late) {
  return (int64_t)born < (int64_t)a.sinks || (int64_t)born >= late ? ~0u : order_of(w);
}

// Copies pairs number first, first + step ..., kAhead of them at a time. D / 8 lanes copy a key, as many its
// value, 16 bytes each; the first of them what is kept about it. pair(m): places from and to.
// pages: the sequence's, in memory or LDS.
template <int D, int kAhead, class Page, class Pair>
__device__ inline void copy_pairs(const EvictArgs& a, const Page* pages, uint32_t head, uint32_t moves, uint32_t group,
                                  uint32_t groups, const Pair& pair) {
  constexpr uint32_t kLanes = D / 8, kTeam = 2 * kLanes;
  const uint32_t teams = blockDim.x / kTeam, team = threadIdx.x / kTeam, in = threadIdx.x % kTeam;
  const int which = in >= kLanes;
  const uint32_t mask = (1u << a.page_log2) - 1;
  uint8_t* const base = a.base[which] + (int64_t)head * a.head[which] + (in - which * kLanes) * 16;
  const int64_t page_stride = a.page[which], place_stride = a.place[which];
  for (uint32_t m0 = group * teams * kAhead + team; m0 < moves; m0 += groups * teams * kAhead) {
    uint32_t from[kAhead], to[kAhead], src[kAhead], dst[kAhead];
    u32x4v data[kAhead];
    float w[kAhead];
    int32_t b[kAhead];
    bool live[kAhead];
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      const uint32_t m = m0 + r * teams;
      live[r] = m < moves;
      const uint2 p = pair(live[r] ? m : m0);
      from[r] = p.x;
      to[r] = p.y;
    }
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      src[r] = (uint32_t)pages[from[r] >> a.page_log2];
      dst[r] = (uint32_t)pages[to[r] >> a.page_log2];
    }
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      live[r] = live[r] && src[r] < a.n_pages && dst[r] < a.n_pages;
      if (!live[r]) continue;
      data[r] = *reinterpret_cast<const u32x4v*>(base + (int64_t)src[r] * page_stride +
                                                 (int64_t)(from[r] & mask) * place_stride);
      if (in == 0) {
        const uint64_t at = ((uint64_t)src[r] * a.kv_heads + head) << a.page_log2 | (from[r] & mask);
        w[r] = a.weights[at];
        b[r] = a.born[at];
      }
    }
#pragma unroll
    for (int r = 0; r < kAhead; ++r) {
      if (!live[r]) continue;
      *reinterpret_cast<u32x4v*>(base + (int64_t)dst[r] * page_stride + (int64_t)(to[r] & mask) * place_stride) = data[r];
      if (in == 0) {
        const uint64_t at = ((uint64_t)dst[r] * a.kv_heads + head) << a.page_log2 | (to[r] & mask);
        a.weights_out[at] = w[r];
        a.born_out[at] = b[r];
      }
    }
  }
}

// The counts of a round, from the largest bin down: which one the `left`-th key is in, how many of it are kept
// (left again), and how many it has. By a wave for itself, four bins a lane.
struct Found {
  uint32_t bin, count;
};
__device__ inline Found bin_of(const uint32_t* bins, uint32_t* left) {
  const uint32_t lane = threadIdx.x & 63;
  u32x4v c = (u32x4v)0u;
#pragma unroll
  for (uint32_t i = 0; i < kCopies; ++i) c += *reinterpret_cast<const u32x4v*>(bins + (i + 1) * kBins - 4 * (lane + 1));
  const uint32_t sum = c[0] + c[1] + c[2] + c[3], upto = wave_scan(sum, SumOp());
  const uint32_t at = uniform((uint32_t)__builtin_ctzll(__ballot(upto >= *left)));
  uint32_t rest = *left - (upto - sum), bin = kBins - 4 * lane - 1, count = c[3];  // of lane `at` these hold
#pragma unroll
  for (int i = 2; i >= 0; --i) {
    const bool on = rest > count && bin == kBins - 4 * lane - (uint32_t)(3 - i);
    rest -= on ? count : 0;
    bin -= on;
    count = on ? c[i] : count;
  }
  auto get = [at](uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, (int)at); };
  *left = get(rest);
  return {get(bin), get(count)};
}

// Adds what a wave's lanes found to a round's counts. Lanes of one bin wait for each other: where it is the same
// for all, it is added to once.
__device__ inline void count_bins(uint32_t* bins, uint32_t bin, bool counts) {
  if (!counts) return;
  const uint32_t copy = threadIdx.x % kCopies * kBins, lead = uniform(bin);
  if (__ballot(bin != lead) == 0) {
    const uint64_t who = __ballot(true);
    if ((threadIdx.x & 63) == (uint32_t)__builtin_ctzll(who)) atomicAdd(&bins[lead], (uint32_t)__popcll(who));
  } else {
    atomicAdd(&bins[copy + bin], 1u);
  }
}

// Exclusive sum over the workgroup; `total` gets the sum. Two barriers.
__device__ inline uint32_t sum_before(uint32_t v, uint32_t* lds, uint32_t* total) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t upto = wave_scan(v, SumOp());
  if (lane == 63) lds[wave] = upto;
  __syncthreads();
  uint32_t before = 0, all = 0;
  for (uint32_t w = 0; w < blockDim.x / 64; ++w) {
    if (w == wave) before = all;
    all += lds[w];
  }
  __syncthreads();
  *total = all;
  return before + upto - v;
}

// Longer sequences than LDS holds: a run of keys for each wave, read again for each count.
constexpr int kBatch = 8;  // loads of a kind that go out together

// Calls each(i, rank, whether there is such a key) for keys i = from + `step` times 0, 1 ... + `lane`, in order,
// while from + `step` times that is below `end`. (from, step, end: the same for all that call together.)
template <class Each>
__device__ inline void each_rank(const EvictArgs& a, const int32_t* pages, uint32_t head, int64_t late, uint32_t from,
                                 uint32_t step, uint32_t lane, uint32_t end, const Each& each) {
#pragma unroll 1
  for (uint64_t i0 = from; i0 < end; i0 += (uint64_t)step * kBatch) {
    uint64_t at[kBatch];
    float w[kBatch];
    int32_t b[kBatch];
#pragma unroll
    for (int r = 0; r < kBatch; ++r) {
      const uint64_t i = i0 + (uint64_t)r * step + lane;
      at[r] = (uint32_t)pages[(i < end ? i : i0) >> a.page_log2];
    }
#pragma unroll
    for (int r = 0; r < kBatch; ++r) {
      const uint64_t i = i0 + (uint64_t)r * step + lane;
      at[r] = i < end && at[r] < a.n_pages ? (at[r] * a.kv_heads + head) << a.page_log2 | (i & ((1u << a.page_log2) - 1))
                                           : ~0ull;
      w[r] = a.weights[at[r] != ~0ull ? at[r] : 0];
      b[r] = a.born[at[r] != ~0ull ? at[r] : 0];
    }
#pragma unroll
    for (int r = 0; r < kBatch; ++r) {
      const uint64_t i = i0 + (uint64_t)r * step + lane;
      each((uint32_t)i, at[r] != ~0ull ? rank_of(a, w[r], b[r], late) : 0, i < end);
    }
  }
}

__device__ void select_long(const EvictArgs& a, const int32_t* pages, uint32_t head, uint32_t keys, int64_t late,
                            uint2* out, uint32_t* bins, uint32_t* lds_sum, uint32_t* moves) {
  const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), keep = a.keep;
  uint32_t known = 0, known_mask = 0, left = keep;
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    uint32_t* const mine = bins + shift / 8 * kRound;
    each_rank(a, pages, head, late, 0, kThreads, threadIdx.x, keys, [&](uint32_t, uint32_t r, bool there) {
      count_bins(mine, (r >> shift) & 255, there && (r & known_mask) == known);
    });
    __syncthreads();
    known |= bin_of(mine, &left).bin << shift;
    known_mask |= 255u << shift;
  }
  const uint32_t per = ((keys + kWaves - 1) / kWaves + 63) & ~63u;
  const uint32_t from = wave * per < keys ? wave * per : keys, to = from + per < keys ? from + per : keys;
  auto before = [&](bool on) {  // lanes before this one, and all
    const uint64_t who = __ballot(on);
    return uint2{__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0)),
                 (uint32_t)__popcll(who)};
  };
  // a wave's count, and all before it
  auto before_wave = [&](uint32_t count, uint32_t* all) {
    return uniform(sum_before(lane == 0 ? count : 0, lds_sum, all));
  };
  uint32_t same = 0, all;
  each_rank(a, pages, head, late, from, 64, lane, to,
            [&](uint32_t, uint32_t r, bool there) { same += before(there && r == known).y; });
  const uint32_t same_before = before_wave(same, &all);
  auto flag = [&](uint32_t i, uint32_t r, bool there) {  // of a place that comes free, or a key that moves
    const bool equal = there && r == known;
    const uint2 n = before(equal);
    const bool kept = r > known || (equal && same + n.x < left);
    same += n.y;
    return there && kept != (i < keep);
  };
  uint32_t count = 0;
  same = same_before;
  each_rank(a, pages, head, late, from, 64, lane, to,
            [&](uint32_t i, uint32_t r, bool there) { count += before(flag(i, r, there)).y; });
  uint32_t at = before_wave(count, &all);
  *moves = all / 2;  // free places all lie before keep, moving keys behind: as many of both
  same = same_before;
  each_rank(a, pages, head, late, from, 64, lane, to, [&](uint32_t i, uint32_t r, bool there) {
    const bool on = flag(i, r, there);
    const uint2 n = before(on);
    if (on && i < keep) out[at + n.x].y = i;
    if (on && i >= keep) out[at + n.x - *moves].x = i;
    at += n.y;
  });
}

// How many of the workgroup's keys with a flag come before a thread's key number r, in the keys' order. counts:
// kKeys times the waves, of the workgroup. One barrier.
template <int kKeys>
struct Ordered {
  static constexpr int kEntries = kKeys * kWaves / 64;  // a lane's
  static_assert(kWaves % kEntries == 0, "");
  uint32_t flags;   // of the thread's keys, a bit each
  uint32_t before;  // of the entries number wave % kEntries of each lane's
  uint32_t all;

  __device__ void count(uint32_t* counts) {
    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
    uint32_t mine = 0;
#pragma unroll 4
    for (int r = 0; r < kKeys; ++r) {
      const uint32_t n = (uint32_t)__popcll(__ballot(flags >> r & 1));
      if (lane == (uint32_t)r) mine = n;
    }
    if (lane < kKeys) counts[lane * kWaves + wave] = mine;
    __syncthreads();
    uint32_t sum = 0;
    before = 0;
#pragma unroll
    for (int i = 0; i < kEntries; ++i) {
      if (wave % kEntries == (uint32_t)i) before = sum;
      sum += counts[lane * kEntries + i];
    }
    const uint32_t upto = wave_scan(sum, SumOp());
    all = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    before += upto - sum;
  }
  // (by whole waves)
  __device__ uint32_t of(uint32_t r) const {
    const uint32_t wave = uniform(threadIdx.x >> 6);
    const uint32_t x = (uint32_t)__builtin_amdgcn_readlane((int)before, (int)((r * kWaves + wave) / kEntries));
    const uint64_t who = __ballot(flags >> r & 1);
    return x + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0));
  }
};

template <int D, int kKeys>
__global__ __launch_bounds__(kThreads, kKeys == kNarrowKeys ? 8 : 4) void select_kernel(EvictArgs a) {
  constexpr bool kNarrow = kKeys == kNarrowKeys;
  constexpr int kGroup = kNarrow ? 4 : 8;  // loads of a kind that go out together
  __shared__ __attribute__((aligned(16))) uint32_t rank[kKeys * kThreads], bins[4 * kRound];
  __shared__ uint32_t counts[2][kKeys * kWaves];
  const uint32_t tid = threadIdx.x;
  for (uint32_t pair = blockIdx.x; pair < a.n_seq * a.kv_heads; pair += gridDim.x) {
    const uint32_t s = pair / a.kv_heads, head = pair % a.kv_heads;
    const int32_t* const pages = a.own_pages + (uint64_t)s * a.own_width;
    // the first keys' pages are looked up while the length is on its way
    const uint32_t places = a.own_width << a.page_log2;
    uint32_t page[kGroup];
#pragma unroll
    for (int r = 0; r < kGroup; ++r) {
      const uint32_t i = r * kThreads + tid;
      page[r] = places ? (uint32_t)pages[(i < places ? i : 0) >> a.page_log2] : kNoPage;
    }
    const uint32_t keys = keys_of(a, s), keep = a.keep < keys ? a.keep : keys;
    const int64_t late = (int64_t)a.total[s] - a.recent;
    if (head == 0 && tid == 0) a.len_out[s] = (int32_t)keep;
    for (uint32_t i = tid; i < 4 * kRound; i += kThreads) bins[i] = 0;

    // What stays where it is is written on, and the others' places by who copies pairs. For no key a first one's
    // weight is loaded.
#pragma unroll 1
    for (uint32_t i0 = 0; i0 < keys; i0 += kGroup * kThreads) {
      float w[kGroup];
      int32_t b[kGroup];
      uint64_t at[kGroup];
#pragma unroll
      for (int r = 0; r < kGroup; ++r) {
        const uint32_t i = i0 + r * kThreads + tid;
        at[r] = i < keys && page[r] < a.n_pages
                    ? ((uint64_t)page[r] * a.kv_heads + head) << a.page_log2 | (i & ((1u << a.page_log2) - 1)) : ~0ull;
        w[r] = a.weights[at[r] != ~0ull ? at[r] : 0];
        b[r] = a.born[at[r] != ~0ull ? at[r] : 0];
      }
      if (!kNarrow) {
#pragma unroll
        for (int r = 0; r < kGroup; ++r) {
          const uint32_t i = i0 + (kGroup + r) * kThreads + tid;
          page[r] = (uint32_t)pages[(i < keys ? i : 0) >> a.page_log2];
        }
      }
#pragma unroll
      for (int r = 0; r < kGroup; ++r) {
        const uint32_t i = i0 + r * kThreads + tid;
        const bool there = at[r] != ~0ull, stays = there && i < keep;
        if (i < kKeys * kThreads) rank[i] = there ? rank_of(a, w[r], b[r], late) : 0;
        if (stays && a.weights_out != a.weights) a.weights_out[at[r]] = w[r];
        if (stays && a.born_out != a.born) a.born_out[at[r]] = b[r];
      }
    }
    __syncthreads();
    uint32_t moves = 0;
    uint2* const out = a.pairs + (uint64_t)pair * a.most;
    if (keys <= a.keep || keep == 0) {  // all stay, or none
    } else if (!kNarrow && keys > kKeys * kThreads) {
      select_long(a, pages, head, keys, late, out, bins, counts[0], &moves);
    } else {
      uint32_t known = 0, known_mask = 0, left = keep, same = 0;  // same: keys of the last kept one's rank
#pragma unroll 1
      for (int shift = 24; shift >= 0; shift -= 8) {
        uint32_t* const mine = bins + shift / 8 * kRound;
#pragma unroll 4
        for (uint32_t i0 = 0; i0 < keys; i0 += kThreads) {
          const uint32_t r = rank[i0 + tid];  // (of no key, of none of these bits or not counted)
          count_bins(mine, (r >> shift) & 255, i0 + tid < keys && (r & known_mask) == known);
        }
        __syncthreads();
        const Found found = bin_of(mine, &left);
        known |= found.bin << shift;
        known_mask |= 255u << shift;
        same = found.count;
      }
      const bool all_same = left == same;  // all of them are kept: no need to know which come first
      Ordered<kKeys> order;
      order.flags = 0;
      uint32_t more = 0, there = 0;  // of a larger rank; keys at all
#pragma unroll 4
      for (uint32_t r = 0; r * kThreads < keys; ++r) {
        const uint32_t i = r * kThreads + tid, x = rank[i], is = i < keys ? 1u : 0u;
        there |= is << r;
        order.flags |= (x == known ? is : 0u) << r;
        more |= (x > known ? is : 0u) << r;
      }
      if (!all_same) {
        order.count(counts[0]);
        uint32_t first = 0;
#pragma unroll 1
        for (uint32_t r = 0; r * kThreads < keys; ++r) first |= (order.of(r) < left ? 1u : 0u) << r;
        order.flags &= first;
      }
      const uint32_t kept = more | order.flags;
      uint32_t within = 0;  // places within the budget
#pragma unroll 1
      for (uint32_t r = 0; r * kThreads + tid < keep; ++r) within |= 1u << r;
      order.flags = (kept ^ within) & there;
      order.count(counts[1]);
      moves = order.all / 2;  // free places all lie before keep, moving keys behind: as many of both
      uint16_t* const half = reinterpret_cast<uint16_t*>(rank);
      // (ranks are not needed any more once all have counted)
#pragma unroll 1
      for (uint32_t r = 0; r * kThreads < keys; ++r) {
        const uint32_t i = r * kThreads + tid, at = order.of(r);
        if (!(order.flags >> r & 1)) continue;
        if (kNarrow && a.copies) {
          if (i < keep) half[2 * at + 1] = (uint16_t)i;
          else half[2 * (at - moves)] = (uint16_t)i;
        } else {
          if (i < keep) out[at].y = i;
          else out[at - moves].x = i;
        }
      }
    }
    if (kNarrow && a.copies) {
      __syncthreads();
      copy_pairs<D, 2>(a, pages, head, moves, 0, 1, [&](uint32_t m) { return uint2{rank[m] & 0xffffu, rank[m] >> 16}; });
    } else if (tid == 0) {
      a.moves[pair] = moves;
    }
    __syncthreads();
  }
}

template <int D>
__global__ __launch_bounds__(kMoveThreads) void move_kernel(EvictArgs a) {
  for (uint32_t pair = blockIdx.y; pair < a.n_seq * a.kv_heads; pair += gridDim.y) {
    const uint32_t s = pair / a.kv_heads;
    const uint2* const pairs = a.pairs + (uint64_t)pair * a.most;
    copy_pairs<D, 4>(a, a.own_pages + (uint64_t)s * a.own_width, pair - s * a.kv_heads, a.moves[pair], blockIdx.x, gridDim.x,
                  [&](uint32_t m) { return pairs[m]; });
  }
}

template <int D>
gleam_status launch_evict(const EvictArgs& a, bool narrow, hipStream_t s) {
  const uint32_t n = a.n_seq * a.kv_heads;
  const uint64_t most = max_workgroups(kThreads);
  const dim3 grid((uint32_t)(n < most ? n : most));
  if (narrow) hipLaunchKernelGGL((select_kernel<D, kNarrowKeys>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((select_kernel<D, kWideKeys>), grid, dim3(kThreads), 0, s, a);
  const gleam_status st = launch_status("select_kernel");
  if (st != GLEAM_OK || a.copies || a.most == 0) return st;
  // workgroups for each sequence and head: as many as there may be moves for, and as give kMoveGroups in all
  constexpr uint32_t teams = kMoveThreads / (D / 4);
  const uint32_t want = (a.most + 4 * teams - 1) / (4 * teams), share = kMoveGroups / n;
  const uint32_t x = want < share ? want : share;
  hipLaunchKernelGGL(move_kernel<D>, dim3(x ? x : 1, n < 65535 ? n : 65535), dim3(kMoveThreads), 0, s, a);
  return launch_status("move_kernel");
}

// Pairs of places that a sequence and head can have.
uint64_t most_moves(const gleam_kv_pages* kv, const gleam_evict* in) {
  const uint64_t keys = in->own_width * kv->page_tokens;
  if (keys <= in->keep) return 0;
  return keys - in->keep < in->keep ? keys - in->keep : in->keep;
}

struct EvictWs {
  size_t moves, pairs, bytes;
};
EvictWs evict_ws(const gleam_kv_pages* kv, const gleam_evict* in) {
  const uint64_t n = in->n_seq * kv->kv_heads;
  EvictWs w{};
  w.pairs = (n * 4 + 255) & ~(size_t)255;
  w.bytes = w.pairs + ((n * most_moves(kv, in) * sizeof(uint2) + 255) & ~(size_t)255);
  if (w.bytes == 0) w.bytes = 256;
  return w;
}

gleam_status validate_evict(const gleam_kv_pages* kv, const gleam_evict* in, const char* who) {
  gleam_status st = validate_kv(kv, who);
  if (st != GLEAM_OK) return st;
  if (!in) {
    set_error("%s: null arguments", who);
    return GLEAM_E_INVALID;
  }
  if (in->n_seq > kMostSeq) {
    set_error("%s: more than 2^20 sequences", who);
    return GLEAM_E_UNSUPPORTED;
  }
  if (in->own_width > (uint64_t)INT32_MAX / kv->page_tokens) {
    set_error("%s: a table row of 2^31 keys or more", who);
    return GLEAM_E_INVALID;
  }
  if (in->n_seq * kv->kv_heads > INT32_MAX) {
    set_error("%s: sequences times heads of 2^31 or more", who);
    return GLEAM_E_UNSUPPORTED;
  }
  if (in->n_seq * kv->kv_heads * most_moves(kv, in) > kMostPairs) {
    set_error("%s: more than 2^36 keys that may move", who);
    return GLEAM_E_UNSUPPORTED;
  }
  return GLEAM_OK;
}

}  // namespace

hipError_t preload_kv_evict() {
  hipFuncAttributes attr;
  return hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&move_kernel<128>));
}

}  // namespace gleam

extern "C" size_t gleam_kv_evict_ws_bytes(const gleam_kv_pages* kv, const gleam_evict* in) {
  using namespace gleam;
  clear_error();
  if (validate_evict(kv, in, "gleam_kv_evict") != GLEAM_OK) return 0;
  return evict_ws(kv, in).bytes;
}

extern "C" gleam_status gleam_kv_evict(const gleam_kv_pages* kv, const gleam_evict* in, void* d_ws, size_t ws_bytes,
                                       void* stream) {
  using namespace gleam;
  clear_error();
  const char* const who = "gleam_kv_evict";
  gleam_status st = validate_evict(kv, in, who);
  if (st != GLEAM_OK) return st;
  if ((st = validate_sequences(kv, in->n_seq, in->own_width, in->d_own_pages, in->d_own_len, who)) != GLEAM_OK)
    return st;
  if ((st = validate_places(kv, who)) != GLEAM_OK) return st;
  if (in->n_seq == 0) return GLEAM_OK;
  if (!in->d_total || !in->d_len_out) {
    set_error("%s: null total or len_out", who);
    return GLEAM_E_INVALID;
  }
  const ReadLate reads[] = {{in->d_own_len, 4 * in->n_seq, "own_len"},
                            {in->d_total, 4 * in->n_seq, "total"},
                            {in->d_own_pages, 4 * in->n_seq * in->own_width, "own_pages"}};
  if ((st = validate_len_out(in->d_len_out, in->n_seq, reads, 3, who)) != GLEAM_OK) return st;
  if ((st = validate_tracked(kv, in->d_weights, in->d_weights_out, "weights", who)) != GLEAM_OK) return st;
  if ((st = validate_tracked(kv, in->d_born, in->d_born_out, "born", who)) != GLEAM_OK) return st;
  if (!d_ws || !aligned256(d_ws)) {
    set_error("%s: workspace must be non-null and 256-byte aligned", who);
    return GLEAM_E_INVALID;
  }
  const EvictWs w = evict_ws(kv, in);
  if (ws_bytes < w.bytes) {
    set_error("%s: workspace of %zu bytes, %zu needed", who, ws_bytes, w.bytes);
    return GLEAM_E_WORKSPACE;
  }
  EvictArgs a{};
  a.base[0] = static_cast<uint8_t*>(kv->d_k);
  a.base[1] = static_cast<uint8_t*>(kv->d_v);
  const int64_t* const stride[2] = {kv->k_stride, kv->v_stride};
  for (int i = 0; i < 2; ++i) {
    a.page[i] = 2 * stride[i][0];
    a.place[i] = 2 * stride[i][1];
    a.head[i] = 2 * stride[i][2];
  }
  a.own_pages = in->d_own_pages;
  a.own_len = in->d_own_len;
  a.weights = in->d_weights;
  a.born = in->d_born;
  a.total = in->d_total;
  a.weights_out = in->d_weights_out;
  a.born_out = in->d_born_out;
  a.len_out = in->d_len_out;
  a.moves = reinterpret_cast<uint32_t*>(d_ws);
  a.pairs = reinterpret_cast<uint2*>(static_cast<uint8_t*>(d_ws) + w.pairs);
  a.most = (uint32_t)most_moves(kv, in);
  a.n_seq = (uint32_t)in->n_seq;
  a.own_width = (uint32_t)in->own_width;
  a.page_log2 = (uint32_t)log2_exact(kv->page_tokens);
  a.n_pages = (uint32_t)kv->n_pages;
  a.kv_heads = kv->kv_heads;
  a.keep = in->keep;
  a.sinks = in->sinks;
  a.recent = in->recent;
  const bool narrow = in->own_width * kv->page_tokens <= kNarrowKeys * kThreads;
  a.copies = narrow && in->n_seq * kv->kv_heads >= kManyPairs;
  hipStream_t s = (hipStream_t)stream;
  return kv->head_dim == 64    ? launch_evict<64>(a, narrow, s)
         : kv->head_dim == 128 ? launch_evict<128>(a, narrow, s)
                               : launch_evict<256>(a, narrow, s);
}
