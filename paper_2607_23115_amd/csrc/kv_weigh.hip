// How much attention each key of a paged cache gets: weight[key] += sum over the rows (a token and a query
// head of the key's head) that see it of exp(scale q.k - lse), lse the row's log sum of exponentials from
// the attention itself.
//
// A key's sum needs no other key, so the keys are cut anywhere and nothing is joined afterwards. S^T = K Q^T by
// v_mfma_f32_16x16x32, 16 rows at a time: a lane gets one row's scores with four keys of 16, keeps the sums of
// its keys' exponentials, and the 16 lanes of the same keys add theirs up at the end.
//   few rows   a wave for itself streams through 32 keys at a time, the next 32 on their way during the
//              products. All halves of 64 keys of all sequences and heads are dealt out evenly, in order, so
//              that lengths do not matter. Up to three tiles of rows stay in LDS; more are loaded again for each
//              32 keys, and waited for (64 sequences of 1,500 keys, 5 tiles: 90 us, 3: 45). With few tiles the
//              time is that of reading the keys: 64 sequences of 500 to 4,000, 8 heads of 128, 201 MB in all,
//              37 us (5.4 TB/s; a plain read reaches 7.1), of which 4 to 5 go by before the first keys arrive.
//   many rows  a workgroup keeps 64 keys (of heads of 256, 32) in registers, the same in all waves, and these
//              share the rows. The time is that of the products and the exponentials: a prompt of 4,097
//              tokens, 32 heads on 8 of 128, 91 us (755 TFLOP/s) once the GPU's clocks are up, after some 40 ms
//              of work, and 106 to 117 before, where its products take 28 and the vector instructions 50 of a
//              SIMD's two waves, which overlap in part. Products of one tile under the exponentials of the one
//              before, in one wave, took too many registers (120 us).

#include <type_traits>

#include "gleam_device.h"
#include "kv_device.h"
#include "launch_shape.h"

namespace gleam {
namespace {

constexpr uint32_t kRows = 16;        // rows of a tile
// From this many tiles on the rows are shared by a workgroup's waves: one number for all widths, that at which heads of
// 256 break even. 64 sequences of 1,500 keys, 4 heads of 256, take with 8 tiles 159 us as few rows and 186 as many, with
// 10 192 and 221, with 12 226 and 225, with 14 259 and 250. Narrower heads break even later, and lose some by it: 8
// of 128 with 8 tiles 123 and 165, 10 144 and 175, 12 169 and 179, 14 190 and 192, 16 214 and 195; 8 of 64 83 and 138,
// 97 and 147, 111 and 146, 128 and 157, 152 and 157. One sequence of 4,000 keys, whose keys are few for each wave, a
// whole call: with 8 tiles 15.7 and 15.5, 10 16.3 and 15, 14 19 and 15.
constexpr uint32_t kSplitTiles = 12, kSplitTilesOfOne = 8;
constexpr uint32_t kGroups = 256;     // workgroups: one a CU, and as many waves in it as its registers hold
template <int D> constexpr int kWaves = D == 256 ? 4 : 8;

struct WeighArgs {
  const uint8_t* q;
  int64_t q_token, q_head;  // bytes
  const uint8_t* k;
  int64_t k_page, k_place, k_head;  // bytes
  const int32_t* q_first;
  const int32_t* own_pages;
  const int32_t* own_len;
  const float* lse;
  const float* weights;
  float* weights_out;
  int32_t* born;  // nullable, with positions
  const int32_t* positions;
  uint32_t n_tokens, n_seq, own_width;
  uint32_t q_heads, kv_heads, ratio, page_log2, n_pages;
  uint32_t ratio_mul, ratio_shift;
  uint32_t most_few;  // rows
  float scale_log2;
};

// row / ratio of rows below 2^31: 2 row times 2^(31 + s) / ratio rounded up, 2^s the power of two that ratio is
// not above.
__device__ inline uint32_t token_of(const WeighArgs& a, uint32_t row) {
  return __umulhi(2 * row, a.ratio_mul) >> a.ratio_shift;
}

// A sequence as a wave finds it: of its keys, units of the two kinds for each head.
struct Seq {
  uint32_t first, tokens, keys;
  uint32_t blocks;  // many rows: of kBlock keys
  uint32_t halves;  // few rows: of 32 keys
};

template <int D> constexpr uint32_t kBlock = D == 256 ? 32 : 64;

template <int D>
__device__ inline Seq seq_at(const WeighArgs& a, uint32_t s) {
  Seq r{};
  if (s >= a.n_seq) return r;
  const uint32_t first = (uint32_t)clamp_to(a.q_first[s], (int32_t)a.n_tokens);
  const uint32_t end = (uint32_t)clamp_to(a.q_first[s + 1], (int32_t)a.n_tokens);
  r.first = first;
  r.tokens = end > first ? end - first : 0;
  r.keys = a.n_pages ? (uint32_t)clamp_to(a.own_len[s], (int32_t)(a.own_width << a.page_log2)) : 0;
  if ((uint64_t)r.tokens * a.ratio > a.most_few) r.blocks = (r.keys + kBlock<D> - 1) / kBlock<D>;
  else r.halves = (r.keys + 31) / 32;
  return r;
}

__device__ inline Seq of_lane(const Seq& s, uint32_t i) {
  auto get = [i](uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, (int)i); };
  return {get(s.first), get(s.tokens), get(s.keys), get(s.blocks), get(s.halves)};
}

// The value that the lane kBy further on among the same 16 has, going round.
template <int kBy>
__device__ inline float turned(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x120 + kBy, 0xf, 0xf, false));
}
__device__ inline float sum_of_16(float x) {
  x += turned<8>(x);
  x += turned<4>(x);
  x += turned<2>(x);
  return x + turned<1>(x);
}

// What is added for the lane's four keys of 16 from `key` on to the sums of `acc`. seen: how many keys the
// lane's row sees; masked: whether that matters to any row.
__device__ inline void add_weights(const f32x4& score, float scale, float down, bool masked, uint32_t key, uint32_t seen,
                                   float (&acc)[4]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float p = __builtin_amdgcn_exp2f(fmaf(score[e], scale, down));
    acc[e] += masked && key + e >= seen ? 0.f : p;
  }
}

// How many keys a row sees: none where there is no such row, and none where its lse is +infinity, which leaves it out
// (its scores may be anything then, and exp(NaN - infinity) is not 0).
__device__ inline uint32_t seen_by(const WeighArgs& a, const Seq& seq, uint32_t row, float lse) {
  const int64_t sees = (int64_t)seq.keys - seq.tokens + token_of(a, row) + 1;
  return row < seq.tokens * a.ratio && sees > 0 && lse != INFINITY ? (uint32_t)sees : 0;
}

// Rows are loaded whole, and pass through LDS into the products' layout: loads of 64 bytes of 16 rows, straight
// into it, take the caches four times as many accesses (keys read 15% slower, queries bound many rows).
template <int D>
struct Staged {
  static constexpr uint32_t kPieces = D / 8, kLoadRows = 64 / kPieces;  // 16-byte pieces of a row, rows of a load
  static constexpr int kLoads = 16 / kLoadRows;                         // of 16 rows
  static constexpr uint32_t kTile = 16 * 2 * D;                         // bytes of 16 rows
  static constexpr int kHeld = 3;                                       // tiles of few rows that stay in LDS
  static constexpr uint32_t kBytes = (1 + kHeld) * kTile;               // of a wave
  // rows of one piece each, or of one row all pieces, fall into different banks
  static __device__ uint32_t at(uint32_t row, uint32_t piece) {
    return row * (2 * D) + ((piece ^ (D == 64 ? (row >> 1) & 7 : row & 15)) << 4);
  }
  // What the lane loads of 16 rows goes to row load_row() + i * kLoadRows, piece(). Other lanes of the wave read it:
  // store() keeps the wave's earlier loads from that place before it and the later ones behind it.
  static __device__ uint32_t load_row() { return (threadIdx.x & 63) / kPieces; }
  static __device__ uint32_t piece() { return (threadIdx.x & 63) % kPieces; }
  static __device__ void store(char* lds, const u32x4v (&x)[kLoads]) {
    wave_lds_sync();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) *reinterpret_cast<u32x4v*>(lds + at(i * kLoadRows + load_row(), piece())) = x[i];
    wave_lds_sync();
  }
  // The 32 dims from 32 i on of a row, a lane's eight; from: at(row, lane / 16).
  static __device__ Pack8 read(const char* lds, uint32_t from, int i) {
    Pack8 x;
    x.u = *reinterpret_cast<const u32x4v*>(lds + (from ^ (i << 6)));
    return x;
  }
};

// Rows of a sequence and key head, 16 a tile, on their way.
template <int D>
struct Rows {
  static constexpr int kLoads = Staged<D>::kLoads;
  u32x4v q[kLoads];
  float lse;  // of row lane % 16
  const uint8_t* at[kLoads];
  const float* lse_at;

  // From row `row` on; rows that there are not are the last one again.
  __device__ void find(const WeighArgs& a, const Seq& seq, uint32_t head, uint32_t row) {
    const uint32_t last = seq.tokens * a.ratio - 1;
    auto of = [&](uint32_t r, uint64_t* h) {
      if (r > last) r = last;
      const uint32_t token = token_of(a, r);
      *h = head * a.ratio + (r - token * a.ratio);
      return seq.first + (uint64_t)token;
    };
    uint64_t h;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const uint64_t t = of(row + i * Staged<D>::kLoadRows + Staged<D>::load_row(), &h);
      at[i] = a.q + t * a.q_token + h * a.q_head + Staged<D>::piece() * 16;
    }
    const uint64_t t = of(row + (threadIdx.x & 15), &h);
    lse_at = a.lse + t * a.q_heads + h;
  }
  __device__ void step_back(int64_t q_bytes, int64_t lses) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) at[i] -= q_bytes;
    lse_at -= lses;
  }
  __device__ void load() {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) q[i] = *reinterpret_cast<const u32x4v*>(at[i]);
    lse = *lse_at;
  }
  __device__ void wait() {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) arrived(q[i]);
    arrived(lse);
  }
};

// --------------------------------------------------------------------------------------- //
// few rows
// --------------------------------------------------------------------------------------- //
// Halves [from, to) of a sequence and head. lds: the wave's own.
template <class T, int D>
__device__ __forceinline__ void weigh_few(const WeighArgs& a, const Seq& seq, uint32_t s, uint32_t head, uint32_t from,
                                          uint32_t to, char* lds) {
  typedef Staged<D> St;
  constexpr int kLoads = St::kLoads;
  constexpr int kSteps = D / 32;
  const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int64_t base = (int64_t)seq.keys - seq.tokens;  // the first new token's key
  const uint32_t rows = seq.tokens * a.ratio, tiles = (rows + kRows - 1) / kRows;
  const uint32_t place_mask = (1u << a.page_log2) - 1;
  const int32_t* const pages = a.own_pages + (uint64_t)s * a.own_width;
  const uint8_t* const k_head = a.k + (int64_t)head * a.k_head;
  // which of the 32 keys' sums the lane stores (n < 8): of four keys of 16 those that it has scores of
  const uint32_t mine = 16 * (n >> 2) + 4 * g + (n & 3);

  // the rows of a tile, in the products' layout
  Rows<D> r;
  Pack8 q[kSteps];
  uint32_t seen = 0;  // keys that the lane's row sees
  float down = 0.f;
  const uint32_t from_lds = St::at(n, g);
  if (tiles == 1) {
    r.find(a, seq, head, 0);
    r.load();
    St::store(lds + St::kTile, r.q);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) q[i] = St::read(lds + St::kTile, from_lds, i);
    down = -r.lse * kLog2e;
    seen = seen_by(a, seq, n, r.lse);
  }
  // a few tiles of rows stay in LDS
  float held_down[St::kHeld];
  uint32_t held_seen[St::kHeld];
  const bool held = tiles > 1 && tiles <= St::kHeld;
#pragma unroll
  for (int t = 0; t < St::kHeld; ++t) {
    held_down[t] = 0.f;
    held_seen[t] = 0;
    if (!held || (uint32_t)t >= tiles) continue;
    r.find(a, seq, head, kRows * t);
    r.load();
    St::store(lds + (1 + t) * St::kTile, r.q);
    held_down[t] = -r.lse * kLog2e;
    held_seen[t] = seen_by(a, seq, kRows * t + n, r.lse);
  }

  // pages of 16 keys each, 64 of them ahead, a lane each
  auto pages_from = [&](uint32_t half) {
    const uint32_t key = 32 * half + 16 * lane;
    return key < seq.keys && key < 32 * to ? (uint32_t)pages[key >> a.page_log2] : kNoPage;
  };
  uint32_t page_half = from, ahead = pages_from(from);
  u32x4v kk[2][2][kLoads];
  const uint32_t k_off = St::load_row() * (uint32_t)a.k_place + St::piece() * 16;
  typedef std::integral_constant<int, 0> Even;
  typedef std::integral_constant<int, 1> Odd;
  uint64_t at[2];
  float old[2];
  // Asks for the keys; returns where the lane's sum goes.
  auto load = [&](uint32_t half, auto set_) -> uint64_t {
    constexpr int set = decltype(set_)::value;
    if (half - page_half >= 32) {
      page_half = half;
      ahead = pages_from(half);
      arrived(ahead);
    }
    uint32_t p[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      p[b] = (uint32_t)__builtin_amdgcn_readlane((int)ahead, (int)(2 * (half - page_half) + b));
      // 16 keys lie in one page. They are not kept in the caches: a call reads them once (43 us for 45 where 37 are
      // taken now).
      const Window k = window(k_head + (int64_t)p[b] * a.k_page + (int64_t)((32 * half + 16 * b) & place_mask) * a.k_place,
                              p[b] < a.n_pages);
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        kk[set][b][i] = load_from<u32x4v, true>(k, k_off, (uint32_t)(i * St::kLoadRows) * (uint32_t)a.k_place);
    }
    const uint32_t key = 32 * half + mine, page = n < 4 ? p[0] : p[1];
    return n < 8 && key < seq.keys && page < a.n_pages
               ? ((uint64_t)page * a.kv_heads + head) << a.page_log2 | (key & place_mask) : ~0ull;
  };
  auto load_old = [&](uint64_t to_at, auto set_) {
    constexpr int set = decltype(set_)::value;
    at[set] = to_at;
    old[set] = a.weights[to_at != ~0ull ? to_at : 0];
  };
  // Both sets are on their way most of the time: a set is asked for again as soon as it is in LDS.
  auto add = [&](uint32_t half, auto set_) {
    constexpr int set = decltype(set_)::value;
    float acc[2][4] = {};
    uint64_t next = ~0ull;
    auto products = [&](const char* keys, int b) {
      f32x4 score = (f32x4)0.f;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) score = Mfma<T>::run(get(St::read(keys, from_lds, i), T()), get(q[i], T()), score);
      add_weights(score, a.scale_log2, down, true, 32 * half + 16 * b + 4 * g, seen, acc[b]);
    };
    if (tiles == 1) {
      St::store(lds, kk[set][0]);
      St::store(lds + St::kTile, kk[set][1]);
      next = load(half + 2, set_);
#pragma unroll
      for (int b = 0; b < 2; ++b) products(lds + b * St::kTile, b);
    } else if (held) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        St::store(lds, kk[set][b]);
        if (b == 1) next = load(half + 2, set_);
#pragma unroll
        for (int t = 0; t < St::kHeld; ++t) {
          if ((uint32_t)t >= tiles) continue;
#pragma unroll
          for (int i = 0; i < kSteps; ++i) q[i] = St::read(lds + (1 + t) * St::kTile, from_lds, i);
          down = held_down[t];
          seen = held_seen[t];
          products(lds, b);
        }
      }
    } else {
      // (a tile of rows asked for ahead takes registers that others need: 85 us for 90 with 5 tiles, 47 for 39 with one)
      St::store(lds, kk[set][0]);
      St::store(lds + St::kTile, kk[set][1]);
      for (uint32_t t = 0; t < tiles; ++t) {
        r.find(a, seq, head, kRows * t);
        r.load();
        St::store(lds + 2 * St::kTile, r.q);
        down = -r.lse * kLog2e;
        seen = seen_by(a, seq, kRows * t + n, r.lse);
#pragma unroll
        for (int i = 0; i < kSteps; ++i) q[i] = St::read(lds + 2 * St::kTile, from_lds, i);
#pragma unroll
        for (int b = 0; b < 2; ++b) products(lds + b * St::kTile, b);
      }
      next = load(half + 2, set_);
    }
    float sum = 0.f;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float x = sum_of_16(acc[b][e]);
        if (n == 4 * b + e) sum = x;
      }
    const int64_t young = (int64_t)(32 * half + mine) - base;
    sum += young < 0 ? old[set] : 0.f;
    if (at[set] != ~0ull) {
      a.weights_out[at[set]] = sum;
      if (a.born && young >= 0) a.born[at[set]] = a.positions[seq.first + (uint32_t)young];
    }
    load_old(next, set_);
  };
  // No load is in a branch that does not wait for it, as every use behind the branch would wait for all loads:
  // halves behind the last have no pages, and are asked for in vain.
  arrived(ahead);
  load_old(load(from, Even()), Even());
  load_old(load(from + 1, Odd()), Odd());
  for (uint32_t half = from; half < to; half += 2) {
    add(half, Even());
    if (half + 1 < to) add(half + 1, Odd());
  }
}

// --------------------------------------------------------------------------------------- //
// many rows
// --------------------------------------------------------------------------------------- //
template <class T, int D>
__device__ __forceinline__ void weigh_many(const WeighArgs& a, const Seq& seq, uint32_t s, uint32_t head, uint32_t block,
                                           char* lds) {
  typedef Staged<D> St;
  constexpr int kTiles = kBlock<D> / 16, kSteps = D / 32;
  const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const uint32_t n = lane & 15, g = lane >> 4;
  const uint32_t key0 = block * kBlock<D>;
  const int64_t base = (int64_t)seq.keys - seq.tokens;
  // the lane's own key, whose sum it stores: of 16 keys those four that it has scores of
  const uint32_t own = key0 + 16 * (n >> 2) + 4 * g + (n & 3);
  const bool has = (n >> 2) < kTiles && own < seq.keys;
  const uint32_t page = has ? (uint32_t)a.own_pages[(uint64_t)s * a.own_width + (own >> a.page_log2)] : kNoPage;
  const uint32_t place_mask = (1u << a.page_log2) - 1;
  const bool stored = has && page < a.n_pages;
  const uint64_t to = ((uint64_t)(stored ? page : 0) * a.kv_heads + head) << a.page_log2 | (own & place_mask);
  // The keys come by way of LDS too, each wave bringing some of the rows.
  char* const lds_k = lds + kWaves<D> * St::kTile;
  constexpr int kBring = kTiles * St::kLoads / kWaves<D>;
  u32x4v bring[kBring];
#pragma unroll
  for (int i = 0; i < kBring; ++i) {
    const uint32_t load = wave * kBring + i, t = load / St::kLoads, row = load % St::kLoads * St::kLoadRows;
    uint32_t p = (uint32_t)__builtin_amdgcn_readlane((int)page, (int)(4 * t));
    if (p >= a.n_pages) p = 0;  // not stored
    bring[i] = load_at<u32x4v>(a.k + (int64_t)p * a.k_page + (int64_t)(((key0 + 16 * t) & place_mask) + row) * a.k_place +
                                   (int64_t)head * a.k_head,
                               St::load_row() * (uint32_t)a.k_place + St::piece() * 16);
  }
  const float old = a.weights[to];  // (some weight, where none is needed)
#pragma unroll
  for (int i = 0; i < kBring; ++i) {
    const uint32_t load = wave * kBring + i, t = load / St::kLoads, row = load % St::kLoads * St::kLoadRows;
    *reinterpret_cast<u32x4v*>(lds_k + t * St::kTile + St::at(row + St::load_row(), St::piece())) = bring[i];
  }
  __syncthreads();
  Pack8 k[kTiles][kSteps];
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int i = 0; i < kSteps; ++i) k[t][i] = St::read(lds_k + t * St::kTile, St::at(n, g), i);
  float acc[kTiles][4] = {};
  const uint32_t rows = seq.tokens * a.ratio;
  // the first row that sees the first key; tiles of whole rows that all see all keys: from which one on, and how many
  const uint32_t row_least = key0 <= base ? 0 : (uint32_t)(key0 - base) * a.ratio;
  const int64_t row_all = ((int64_t)key0 + kBlock<D> - 1 - base) * a.ratio;
  const uint32_t tile_all = row_all <= 0 ? 0 : (uint32_t)((row_all + kRows - 1) / kRows);
  const uint32_t tiles_all = rows / kRows > tile_all ? rows / kRows - tile_all : 0;
  // From the last rows to the first that see a key: all blocks of a head that run at a time read the same
  // queries then, from the caches. A wave's tiles are kWaves<D> apart, two are on their way. Where the rows of
  // two such tiles are whole tokens, each lane only steps back over those.
  const int32_t tile_least = (int32_t)(row_least / kRows);
  int32_t tile = (int32_t)((rows - 1) / kRows) - (int32_t)wave;
  constexpr uint32_t kBack = 2 * kWaves<D> * kRows;
  const bool whole = kBack % a.ratio == 0;
  const int64_t back_q = kBack / a.ratio * a.q_token, back_lse = (int64_t)(kBack / a.ratio) * a.q_heads;
  char* const mine = lds + wave * St::kTile;
  const uint32_t from_lds = St::at(n, g);
  Rows<D> r[2];
  auto add = [&](auto set_) {
    constexpr int set = decltype(set_)::value;
    St::store(mine, r[set].q);
    const float lse = r[set].lse, down = -lse * kLog2e;
    if (tile >= 2 * kWaves<D>) {  // otherwise the same again, in vain
      if (whole) r[set].step_back(back_q, back_lse);
      else r[set].find(a, seq, head, (uint32_t)(tile - 2 * kWaves<D>) * kRows);
    }
    r[set].load();
    f32x4 score[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) score[t] = (f32x4)0.f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const Pack8 q = St::read(mine, from_lds, i);
#pragma unroll
      for (int t = 0; t < kTiles; ++t) score[t] = Mfma<T>::run(get(k[t][i], T()), get(q, T()), score[t]);
    }
    if ((uint32_t)tile - tile_all >= tiles_all || __any(lse == INFINITY)) {
      const uint32_t seen = seen_by(a, seq, (uint32_t)tile * kRows + n, lse);
#pragma unroll
      for (int t = 0; t < kTiles; ++t)
        add_weights(score[t], a.scale_log2, down, true, key0 + 16 * t + 4 * g, seen, acc[t]);
    } else {
#pragma unroll
      for (int t = 0; t < kTiles; ++t) add_weights(score[t], a.scale_log2, down, false, 0, 0, acc[t]);
    }
    tile -= kWaves<D>;
  };
  typedef std::integral_constant<int, 0> Even;
  typedef std::integral_constant<int, 1> Odd;
  if (tile >= tile_least) {
    // The last tile may have fewer rows than 16: it is found again where steps go back from it.
    r[0].find(a, seq, head, (uint32_t)tile * kRows);
    r[0].load();
    r[1].find(a, seq, head, (uint32_t)(tile >= kWaves<D> ? tile - kWaves<D> : 0) * kRows);
    r[1].load();
    if (tile >= 2 * kWaves<D>) {
      r[0].find(a, seq, head, (uint32_t)(tile - 2 * kWaves<D>) * kRows);
      r[0].step_back(-back_q, -back_lse);
    }
  }
  while (tile >= tile_least) {
    add(Even());
    if (tile >= tile_least) add(Odd());
  }
  float sum = 0.f;
#pragma unroll
  for (int t = 0; t < kTiles; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float x = sum_of_16(acc[t][e]);
      if (n == 4 * t + e) sum = x;
    }
  float(*const sums)[64] = reinterpret_cast<float(*)[64]>(lds + (kWaves<D> + kTiles) * St::kTile);
  sums[wave][lane] = sum;
  __syncthreads();
  if (wave == 0 && stored) {
    sum = own < base ? old : 0.f;
    float added = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves<D>; ++w) added += sums[w][lane];
    a.weights_out[to] = sum + added;
    if (a.born && own >= base) a.born[to] = a.positions[seq.first + (uint32_t)(own - base)];
  }
  // No barrier: the next call's keys are written once all have read these, and its sums behind its first barrier.
}

// Each wave finds its work by walking over the sequences' lengths, 64 a step.
template <class T, int D>
__global__ __launch_bounds__(64 * kWaves<D>) void weigh_kernel(WeighArgs a) {
  // few rows: kBytes a wave; many: a tile of rows a wave, the keys, and sums
  __shared__ __attribute__((aligned(16))) char lds[kWaves<D> * Staged<D>::kBytes];
  static_assert((kWaves<D> + kBlock<D> / 16) * Staged<D>::kTile + kWaves<D> * 256 <= sizeof(lds), "");
  const uint32_t lane = threadIdx.x & 63;
  uint64_t blocks = 0, halves = 0;
  Seq mine{};
  uint64_t upto_blocks = 0, upto_halves = 0;
  for (uint32_t s0 = 0; s0 < a.n_seq; s0 += 64) {
    mine = seq_at<D>(a, s0 + lane);
    upto_blocks = wave_scan((uint64_t)mine.blocks * a.kv_heads, SumOp());
    upto_halves = wave_scan((uint64_t)mine.halves * a.kv_heads, SumOp());
    blocks += __shfl(upto_blocks, 63, 64);
    halves += __shfl(upto_halves, 63, 64);
  }
  const bool one_step = a.n_seq <= 64;  // what was found still is at hand

  if (blocks) {
    // A prompt's first keys are seen by the most rows. Every other round goes the other way round, so that who
    // has the longest of one gets the shortest of the next.
    uint64_t round = 0, before = 0;
    auto unit_of = [&](uint64_t r) {
      return r * gridDim.x + (r & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
    };
    for (uint32_t s0 = 0; s0 < a.n_seq; s0 += 64) {
      if (!one_step) {
        mine = seq_at<D>(a, s0 + lane);
        upto_blocks = wave_scan((uint64_t)mine.blocks * a.kv_heads, SumOp());
      }
      const uint64_t all = __shfl(upto_blocks, 63, 64);
      for (uint64_t u; (u = unit_of(round)) < before + all; ++round) {
        const uint32_t i = uniform((uint32_t)__builtin_ctzll(__ballot(upto_blocks > u - before)));
        const Seq seq = of_lane(mine, i);
        const uint64_t end = __shfl(upto_blocks, (int)i, 64);
        const uint32_t at = uniform((uint32_t)(u - before - (end - (uint64_t)seq.blocks * a.kv_heads)));
        const uint32_t block = uniform(at / a.kv_heads);
        weigh_many<T, D>(a, seq, s0 + i, at - block * a.kv_heads, block, lds);
      }
      before += all;
    }
    __syncthreads();  // what follows uses the same LDS otherwise
  }
  if (halves) {
    const uint64_t waves = (uint64_t)gridDim.x * kWaves<D>, wave = (uint64_t)blockIdx.x * kWaves<D> + uniform(threadIdx.x >> 6);
    uint64_t from = halves * wave / waves, before = 0;
    const uint64_t to = halves * (wave + 1) / waves;
    for (uint32_t s0 = 0; s0 < a.n_seq && from < to; s0 += 64) {
      if (!one_step) {
        mine = seq_at<D>(a, s0 + lane);
        upto_halves = wave_scan((uint64_t)mine.halves * a.kv_heads, SumOp());
      }
      const uint64_t all = __shfl(upto_halves, 63, 64);
      while (from < to && from < before + all) {
        const uint32_t i = uniform((uint32_t)__builtin_ctzll(__ballot(upto_halves > from - before)));
        const Seq seq = of_lane(mine, i);
        const uint64_t end = __shfl(upto_halves, (int)i, 64);
        const uint32_t at = uniform((uint32_t)(from - before - (end - (uint64_t)seq.halves * a.kv_heads)));
        const uint32_t head = uniform(at / seq.halves), half = at - head * seq.halves;
        uint32_t last = seq.halves;
        if (to - from < last - half) last = half + (uint32_t)(to - from);
        last = uniform(last);
        weigh_few<T, D>(a, seq, s0 + i, head, half, last, lds + uniform(threadIdx.x >> 6) * Staged<D>::kBytes);
        from += last - half;
      }
      before += all;
    }
  }
}

template <class T, int D>
void launch_weigh(const WeighArgs& a, uint64_t halves, hipStream_t s) {
  // no more than there may be with work, where each takes two halves of many rows
  const uint64_t groups = (halves + 1) / 2;
  const uint32_t n = (uint32_t)(groups < kGroups ? groups : kGroups);
  hipLaunchKernelGGL((weigh_kernel<T, D>), dim3(n), dim3(64 * kWaves<D>), 0, s, a);
}

}  // namespace

hipError_t preload_kv_weigh() {
  hipFuncAttributes attr;
  return hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&weigh_kernel<Bf16, 128>));
}

gleam_status validate_tracked(const gleam_kv_pages* kv, const void* in, const void* out, const char* name,
                              const char* who) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(in), y = reinterpret_cast<uintptr_t>(out);
  if (kv->n_pages > 0 && (!in || !out || (x & 3) || (y & 3))) {
    set_error("%s: %s must be non-null and 4-byte aligned", who, name);
    return GLEAM_E_INVALID;
  }
  const unsigned __int128 bytes = (unsigned __int128)kv->n_pages * kv->kv_heads * kv->page_tokens * 4;
  if (x != y && (x < y ? y - x : x - y) < bytes) {
    set_error("%s: %s and what it becomes must be the same or not overlap", who, name);
    return GLEAM_E_INVALID;
  }
  return GLEAM_OK;
}

}  // namespace gleam

extern "C" gleam_status gleam_kv_weigh(const gleam_kv_pages* kv, const gleam_weigh* in, void* stream) {
  using namespace gleam;
  clear_error();
  const char* const who = "gleam_kv_weigh";
  gleam_status st = validate_kv(kv, who);
  if (st != GLEAM_OK) return st;
  if (!in) {
    set_error("%s: null arguments", who);
    return GLEAM_E_INVALID;
  }
  if (in->q_heads == 0 || in->q_heads % kv->kv_heads != 0 || in->q_heads > 65535) {
    set_error("%s: q_heads must be a multiple of kv_heads, up to 65535", who);
    return GLEAM_E_INVALID;
  }
  if (kv->k_stride[1] >= 1 << 26) {  // places of 16 keys are reached by 32-bit offsets
    set_error("%s: places of a page 2^26 elements apart or more", who);
    return GLEAM_E_UNSUPPORTED;
  }
  if (in->n_tokens > (uint64_t)INT32_MAX / in->q_heads) {
    set_error("%s: n_tokens * q_heads of 2^31 or more", who);
    return GLEAM_E_UNSUPPORTED;
  }
  if ((st = validate_sequences(kv, in->n_seq, in->own_width, in->d_own_pages, in->d_own_len, who)) != GLEAM_OK)
    return st;
  if (in->n_seq == 0 || kv->n_pages == 0 || in->own_width == 0) return GLEAM_OK;
  if (in->n_tokens > 0 && (st = validate_heads(in->d_q, in->q_stride, "q", who)) != GLEAM_OK) return st;
  if (!in->d_q_first || (in->n_tokens > 0 && !in->d_lse)) {
    set_error("%s: null q_first or lse", who);
    return GLEAM_E_INVALID;
  }
  if ((st = validate_tracked(kv, in->d_weights, in->d_weights_out, "weights", who)) != GLEAM_OK) return st;
  if (!in->d_born != !in->d_positions || (reinterpret_cast<uintptr_t>(in->d_born) & 3)) {
    set_error("%s: born and positions go together, born 4-byte aligned", who);
    return GLEAM_E_INVALID;
  }
  WeighArgs a{};
  a.q = static_cast<const uint8_t*>(in->d_q);
  a.q_token = 2 * in->q_stride[0];
  a.q_head = 2 * in->q_stride[1];
  a.k = static_cast<const uint8_t*>(kv->d_k);
  a.k_page = 2 * kv->k_stride[0];
  a.k_place = 2 * kv->k_stride[1];
  a.k_head = 2 * kv->k_stride[2];
  a.q_first = in->d_q_first;
  a.own_pages = in->d_own_pages;
  a.own_len = in->d_own_len;
  a.lse = in->d_lse;
  a.weights = in->d_weights;
  a.weights_out = in->d_weights_out;
  a.born = in->d_born;
  a.positions = in->d_positions;
  a.n_tokens = (uint32_t)in->n_tokens;
  a.n_seq = (uint32_t)in->n_seq;
  a.own_width = (uint32_t)in->own_width;
  a.q_heads = in->q_heads;
  a.kv_heads = kv->kv_heads;
  a.ratio = in->q_heads / kv->kv_heads;
  while (1u << a.ratio_shift < a.ratio) ++a.ratio_shift;
  a.ratio_mul = (uint32_t)((1ull << (31 + a.ratio_shift)) / a.ratio + 1);
  a.page_log2 = (uint32_t)log2_exact(kv->page_tokens);
  a.n_pages = (uint32_t)kv->n_pages;
  // (fewer sequences times heads than CUs are like one sequence)
  a.most_few = kRows * ((in->n_seq * kv->kv_heads < kGroups ? kSplitTilesOfOne : kSplitTiles) - 1);
  a.scale_log2 = in->scale * kLog2e;
  const uint64_t halves = in->n_seq * kv->kv_heads * ((in->own_width * kv->page_tokens + 31) / 32);
  hipStream_t s = (hipStream_t)stream;
  if (kv->dtype == GLEAM_FP16) {
    kv->head_dim == 64    ? launch_weigh<Fp16, 64>(a, halves, s)
    : kv->head_dim == 128 ? launch_weigh<Fp16, 128>(a, halves, s)
                          : launch_weigh<Fp16, 256>(a, halves, s);
  } else {
    kv->head_dim == 64    ? launch_weigh<Bf16, 64>(a, halves, s)
    : kv->head_dim == 128 ? launch_weigh<Bf16, 128>(a, halves, s)
                          : launch_weigh<Bf16, 256>(a, halves, s);
  }
  return launch_status("weigh_kernel");
}
