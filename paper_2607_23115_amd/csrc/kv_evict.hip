// Keeping a paged cache within a budget: of each sequence's keys, those of a head that gathered the least
// attention make room. Each key head chooses for itself, all keep as many, so the page table and the
// length hold for all heads.
//
// The order of a sequence's keys means nothing to attention (positions are rotated into the keys, and the
// next tokens' keys come behind), so nothing is shifted: kept keys that lie behind the budget move into the
// places within it that come free, the i-th such key into the i-th such place. A sequence a few tokens over
// its budget moves a few keys, not all of them, and no place that is read is written.
//
// select_kernel, a workgroup for each sequence and head: weights as integers in their order, the weight of
// the last key kept found in three rounds of counting 11, 11 and 10 bits, then two running counts in the
// keys' order: of the keys of just that weight, to keep the first ones, and of places that come free and
// keys that move. move_kernel copies the pairs.

#include "kv_device.h"
#include "launch_shape.h"

namespace gleam {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMoveThreads = 256;
constexpr uint32_t kBins = 2048;
// Weights of up to this many keys are kept in LDS between the rounds; of more they are read again.
constexpr uint32_t kLdsKeys = 32768;
constexpr uint32_t kMoveGroups = 2048;  // of move_kernel

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
  uint32_t n_seq, own_width, page_log2, n_pages, kv_heads, keep, sinks, recent;
  uint32_t lds_keys;
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

// A larger number for a larger weight: 0 for NaN, -0 as 0.
__device__ inline uint32_t order_of(float w) {
  const uint32_t b = __float_as_uint(w + 0.f);
  return w != w ? 0 : b ^ ((b >> 31) ? ~0u : 0x80000000u);
}

// Of key i; ~0 for one that is kept whatever its weight.
__device__ inline uint32_t rank_of(const EvictArgs& a, const int32_t* pages, uint32_t head, uint32_t i, int64_t late) {
  const uint64_t at = tracked_at(a, pages, head, i);
  if (at == ~0ull) return 0;
  const float w = a.weights[at];
  const int64_t born = a.born[at];
  return born < (int64_t)a.sinks || born >= late ? ~0u : order_of(w);
}

// Exclusive sum over the workgroup; `total` gets the sum. Two barriers.
__device__ inline uint32_t sum_before(uint32_t v, uint32_t* lds, uint32_t* total) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t upto = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t x = __shfl_up(upto, d, 64);
    if ((int)lane >= d) upto += x;
  }
  if (lane == 63) lds[wave] = upto;
  __syncthreads();
  uint32_t before = 0, all = 0;
#pragma unroll
  for (uint32_t w = 0; w < kWaves; ++w) {
    if (w == wave) before = all;
    all += lds[w];
  }
  __syncthreads();
  *total = all;
  return before + upto - v;
}

__global__ __launch_bounds__(kThreads) void select_kernel(EvictArgs a) {
  extern __shared__ uint32_t lds_rank[];
  __shared__ uint32_t bins[kBins];
  __shared__ uint32_t lds_sum[kWaves], lds_found[2];
  const uint32_t tid = threadIdx.x;
  for (uint32_t pair = blockIdx.x; pair < a.n_seq * a.kv_heads; pair += gridDim.x) {
    const uint32_t s = pair / a.kv_heads, head = pair % a.kv_heads;
    const int32_t* const pages = a.own_pages + (uint64_t)s * a.own_width;
    const uint32_t keys = keys_of(a, s), keep = a.keep < keys ? a.keep : keys;
    const int64_t late = (int64_t)a.total[s] - a.recent;
    if (keys <= a.keep || keep == 0) {  // all stay, or none
      for (uint32_t i = tid; i < keep; i += kThreads) {
        const uint64_t at = tracked_at(a, pages, head, i);
        if (at == ~0ull) continue;
        if (a.weights_out != a.weights) a.weights_out[at] = a.weights[at];
        if (a.born_out != a.born) a.born_out[at] = a.born[at];
      }
      if (tid == 0) a.moves[pair] = 0;
      continue;
    }
    const bool in_lds = keys <= a.lds_keys;
    if (in_lds) {
      for (uint32_t i = tid; i < keys; i += kThreads) lds_rank[i] = rank_of(a, pages, head, i, late);
    }
    auto rank_at = [&](uint32_t i) { return in_lds ? lds_rank[i] : rank_of(a, pages, head, i, late); };

    // the rank of the last one kept: its bits from the top, and how many of the keys that have them are kept
    uint32_t known = 0, known_mask = 0, left = keep;
#pragma unroll
    for (int round = 0; round < 3; ++round) {
      const int shift = round == 0 ? 21 : round == 1 ? 10 : 0;
      const uint32_t mask = round == 2 ? 1023u : 2047u;
      for (uint32_t b = tid; b < kBins; b += kThreads) bins[b] = 0;
      __syncthreads();
      for (uint32_t i0 = 0; i0 < keys; i0 += kThreads) {
        const uint32_t i = i0 + tid;
        uint32_t r = 0;
        bool counts = i < keys;
        if (counts) {
          r = rank_at(i);
          counts = (r & known_mask) == known;
        }
        const uint32_t bin = (r >> shift) & mask;
        // equal bins of a wave would wait for each other: those of its first key are added as one
        const uint64_t who = __ballot(counts);
        if (!who) continue;
        const uint32_t lead = (uint32_t)__builtin_ctzll(who);
        const bool with_lead = counts && bin == __shfl(bin, (int)lead, 64);
        const uint64_t together = __ballot(with_lead);
        if ((tid & 63) == lead) atomicAdd(&bins[bin], (uint32_t)__popcll(together));
        else if (counts && !with_lead) atomicAdd(&bins[bin], 1u);
      }
      __syncthreads();
      // bins from the largest down, two a thread: the one that the last kept key is in
      const uint32_t hi = kBins - 1 - 2 * tid, c0 = bins[hi], c1 = bins[hi - 1];
      uint32_t all;
      const uint32_t before = sum_before(c0 + c1, lds_sum, &all);
      if (before < left && left <= before + c0) {
        lds_found[0] = hi;
        lds_found[1] = left - before;
      } else if (before + c0 < left && left <= before + c0 + c1) {
        lds_found[0] = hi - 1;
        lds_found[1] = left - before - c0;
      }
      __syncthreads();
      known |= lds_found[0] << shift;
      known_mask |= mask << shift;
      left = lds_found[1];
    }

    // a run of keys for each thread: how many of just that rank come before, then free places and moving keys
    const uint32_t per = (keys + kThreads - 1) / kThreads;
    const uint32_t from = tid * per < keys ? tid * per : keys, to = from + per < keys ? from + per : keys;
    uint32_t same = 0, all;
    for (uint32_t i = from; i < to; ++i) same += rank_at(i) == known;
    const uint32_t same_before = sum_before(same, lds_sum, &all);
    uint32_t count = 0;
    same = same_before;
    for (uint32_t i = from; i < to; ++i) {
      const uint32_t r = rank_at(i);
      const bool kept = r > known || (r == known && same++ < left);
      count += i < keep ? !kept : kept;
    }
    // free places all lie before keep, moving keys behind: the sum before a thread is that of the former,
    // then all of those and the latter
    uint32_t at = sum_before(count, lds_sum, &all);
    const uint32_t moves = all / 2;  // as many of both
    uint2* const out = a.pairs + (uint64_t)pair * a.most;
    same = same_before;
    for (uint32_t i = from; i < to; ++i) {
      const uint32_t r = rank_at(i);
      const bool kept = r > known || (r == known && same++ < left);
      if (i < keep ? !kept : kept) {
        if (i < keep) out[at++].y = i;
        else out[at++ - moves].x = i;
      }
    }
    if (a.weights_out != a.weights || a.born_out != a.born) {
      // what stays where it is; move_kernel writes the others' places
      __syncthreads();
      for (uint32_t i = tid; i < keep; i += kThreads) {
        const uint64_t where = tracked_at(a, pages, head, i);
        if (where == ~0ull) continue;
        if (a.weights_out != a.weights) a.weights_out[where] = a.weights[where];
        if (a.born_out != a.born) a.born_out[where] = a.born[where];
      }
    }
    if (tid == 0) a.moves[pair] = moves;
    __syncthreads();
  }
}

// D / 8 lanes copy a key, as many its value, 16 bytes each; the first of them what is kept about it.
template <int D>
__global__ __launch_bounds__(kMoveThreads) void move_kernel(EvictArgs a) {
  constexpr uint32_t kLanes = D / 8, kTeam = 2 * kLanes, kTeams = kMoveThreads / kTeam;
  constexpr uint32_t kAhead = 4;
  const uint32_t team = threadIdx.x / kTeam, in = threadIdx.x % kTeam;
  const int which = in >= kLanes;
  const uint32_t mask = (1u << a.page_log2) - 1;
  for (uint32_t pair = blockIdx.y; pair < a.n_seq * a.kv_heads; pair += gridDim.y) {
    const uint32_t s = pair / a.kv_heads, head = pair % a.kv_heads;
    if (blockIdx.x == 0 && head == 0 && threadIdx.x == 0) {
      const uint32_t keys = keys_of(a, s);
      a.len_out[s] = (int32_t)(keys < a.keep ? keys : a.keep);
    }
    const uint32_t moves = a.moves[pair];
    const int32_t* const pages = a.own_pages + (uint64_t)s * a.own_width;
    const uint2* const pairs = a.pairs + (uint64_t)pair * a.most;
    uint8_t* const base = a.base[which] + (int64_t)head * a.head[which] + (in - which * kLanes) * 16;
    for (uint32_t m0 = blockIdx.x * kTeams * kAhead + team; m0 < moves; m0 += gridDim.x * kTeams * kAhead) {
      u32x4v data[kAhead];
      int64_t to[kAhead];
      float w[kAhead];
      int32_t b[kAhead];
      uint64_t tracked[kAhead];
      bool live[kAhead];
#pragma unroll
      for (uint32_t r = 0; r < kAhead; ++r) {
        const uint32_t m = m0 + r * kTeams;
        live[r] = false;
        if (m >= moves) continue;
        const uint2 p = pairs[m];
        const uint32_t src = (uint32_t)pages[p.x >> a.page_log2], dst = (uint32_t)pages[p.y >> a.page_log2];
        live[r] = src < a.n_pages && dst < a.n_pages;
        if (!live[r]) continue;
        data[r] = *reinterpret_cast<const u32x4v*>(base + (int64_t)src * a.page[which] +
                                                   (int64_t)(p.x & mask) * a.place[which]);
        to[r] = (int64_t)dst * a.page[which] + (int64_t)(p.y & mask) * a.place[which];
        if (in == 0) {
          const uint64_t at = ((uint64_t)src * a.kv_heads + head) << a.page_log2 | (p.x & mask);
          tracked[r] = ((uint64_t)dst * a.kv_heads + head) << a.page_log2 | (p.y & mask);
          w[r] = a.weights[at];
          b[r] = a.born[at];
        }
      }
#pragma unroll
      for (uint32_t r = 0; r < kAhead; ++r) {
        if (!live[r]) continue;
        *reinterpret_cast<u32x4v*>(base + to[r]) = data[r];
        if (in == 0) {
          a.weights_out[tracked[r]] = w[r];
          a.born_out[tracked[r]] = b[r];
        }
      }
    }
  }
}

constexpr uint64_t kMostPairs = 1ull << 36;

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
  return hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&select_kernel));
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
  const uint64_t keys = in->own_width * kv->page_tokens;
  a.lds_keys = keys < kLdsKeys ? (uint32_t)keys : kLdsKeys;
  hipStream_t s = (hipStream_t)stream;
  const uint32_t n = a.n_seq * a.kv_heads;
  const uint32_t most = (uint32_t)max_workgroups(kThreads);
  hipLaunchKernelGGL(select_kernel, dim3(n < most ? n : most), dim3(kThreads), a.lds_keys * 4, s, a);
  if ((st = launch_status("select_kernel")) != GLEAM_OK) return st;
  // workgroups for each sequence and head: as many as there may be moves for, and as give kMoveGroups in all
  const uint32_t teams = kMoveThreads / (kv->head_dim / 4);
  const uint32_t want = (a.most + 4 * teams - 1) / (4 * teams), share = kMoveGroups / n;
  const uint32_t x = want < share ? want : share;
  const dim3 grid(x ? x : 1, n < 65535 ? n : 65535);
  if (kv->head_dim == 64) hipLaunchKernelGGL(move_kernel<64>, grid, dim3(kMoveThreads), 0, s, a);
  else if (kv->head_dim == 128) hipLaunchKernelGGL(move_kernel<128>, grid, dim3(kMoveThreads), 0, s, a);
  else hipLaunchKernelGGL(move_kernel<256>, grid, dim3(kMoveThreads), 0, s, a);
  return launch_status("move_kernel");
}
