// How much attention each key of a paged cache gets: weight[key] += sum over the rows (a token and a query
// head of the key's head) that see it of exp(scale q.k - lse), lse the row's log sum of exponentials from
// the attention itself.
//
// A key's sum needs no other key, so keys are cut into units of any size and nothing is joined afterwards:
// a wave holds 64 keys in registers (of heads of 256, 32) as the row operand of v_mfma_f32_16x16x32, S^T = K
// Q^T, and walks 16 rows at a time; a lane keeps the sums of its scores' keys, and the 16 lanes of the same
// keys add theirs up at the end. With few rows the time is that of reading the keys, with many that of the
// products and the exponentials.

#include "kv_device.h"
#include "launch_shape.h"

namespace gleam {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr uint32_t kRows = 16;          // rows of a tile
constexpr uint32_t kSplitTiles = 8;     // from this many tiles on a workgroup's waves share keys and split the rows
constexpr uint32_t kMostGroups = 512;   // workgroups: two a CU

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
  float scale_log2;
};

// A sequence as a workgroup finds it.
struct Seq {
  uint32_t first, tokens, keys;
  uint32_t units;  // a head's
};

// The keys of a unit: a wave's own 64 for each wave, or the same 64 for all.
template <int D> constexpr uint32_t kWaveKeys = D == 256 ? 32 : 64;

__device__ inline bool splits_rows(uint32_t tokens, uint32_t ratio) {
  return (uint64_t)tokens * ratio > kRows * (kSplitTiles - 1);
}

template <int D>
__device__ inline Seq seq_at(const WeighArgs& a, uint32_t s) {
  Seq r{};
  const uint32_t first = (uint32_t)clamp_to(a.q_first[s], (int32_t)a.n_tokens);
  const uint32_t end = (uint32_t)clamp_to(a.q_first[s + 1], (int32_t)a.n_tokens);
  r.first = first;
  r.tokens = end > first ? end - first : 0;
  r.keys = a.n_pages ? (uint32_t)clamp_to(a.own_len[s], (int32_t)(a.own_width << a.page_log2)) : 0;
  const uint32_t per = splits_rows(r.tokens, a.ratio) ? kWaveKeys<D> : kWaves * kWaveKeys<D>;
  r.units = (r.keys + per - 1) / per;
  return r;
}

// The value that the lane `by` further on among the same 16 has, going round.
template <int kBy>
__device__ inline float turned(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x120 + kBy, 0xf, 0xf, false));
}

template <class T, int D>
__device__ __forceinline__ void weigh_unit(const WeighArgs& a, const Seq& seq, uint32_t s, uint32_t head, uint32_t unit,
                                           float (*lds)[64]) {
  constexpr uint32_t kKeys = kWaveKeys<D>;
  constexpr int kTiles = kKeys / 16, kSteps = D / 32;
  const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const uint32_t n = lane & 15, g = lane >> 4;
  const bool split = splits_rows(seq.tokens, a.ratio);
  const uint32_t key0 = (split ? unit : unit * kWaves + wave) * kKeys;
  const int64_t base = (int64_t)seq.keys - seq.tokens;  // the first new token's key
  // the lane's own key, whose sum it stores: 4 g + its place among four of the 16 keys that n / 4 names
  const uint32_t own = key0 + 16 * (n >> 2) + 4 * g + (n & 3);
  const bool has = (n >> 2) < kTiles && own < seq.keys;
  const int32_t* const pages = a.own_pages + (uint64_t)s * a.own_width;
  const uint32_t page = has ? (uint32_t)pages[own >> a.page_log2] : kNoPage;
  const uint32_t place_mask = (1u << a.page_log2) - 1;

  if (key0 < seq.keys) {
    Pack8 k[kTiles][kSteps];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      // 16 keys lie in one page; those that are none are of page 0, and their sums are not stored
      uint32_t p = (uint32_t)__builtin_amdgcn_readlane((int)page, 4 * t);
      if (p >= a.n_pages) p = 0;
      const uint8_t* const at = a.k + (int64_t)p * a.k_page + (int64_t)((key0 + 16 * t) & place_mask) * a.k_place +
                                (int64_t)head * a.k_head + n * a.k_place + g * 16;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) k[t][i].u = *reinterpret_cast<const u32x4v*>(at + i * 64);
    }
    const bool stored = has && page < a.n_pages;
    const uint64_t to = ((uint64_t)page * a.kv_heads + head) << a.page_log2 | (own & place_mask);
    float sum = 0.f;
    const bool is_new = own >= base;
    if (stored && !is_new && !(split && wave > 0)) sum = a.weights[to];

    float acc[kTiles][4];
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[t][e] = 0.f;
    // the first row that sees the first key
    const uint32_t rows = seq.tokens * a.ratio;
    const uint32_t row_least = key0 <= base ? 0 : (uint32_t)(key0 - base) * a.ratio;
    const uint32_t step = split ? kWaves * kRows : kRows;
    const uint32_t step_tokens = step / a.ratio, step_rest = step % a.ratio;
    uint32_t row0 = row_least / kRows * kRows + (split ? wave * kRows : 0);
    uint32_t token = (row0 + n) / a.ratio, in_head = (row0 + n) % a.ratio;

    Pack8 q[kSteps];
    float bias;
    auto load = [&]() {
      const bool live = row0 + n < rows;
      const uint64_t t = seq.first + (live ? token : 0), h = head * a.ratio + in_head;
      const uint8_t* const at = a.q + t * a.q_token + h * a.q_head + g * 16;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) q[i].u = *reinterpret_cast<const u32x4v*>(at + i * 64);
      bias = a.lse[t * a.q_heads + h];
    };
    if (row0 < rows) load();
    while (row0 < rows) {
      f32x4 score[kTiles];
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        score[t] = (f32x4)0.f;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) score[t] = Mfma<T>::run(get(k[t][i], T()), get(q[i], T()), score[t]);
      }
      const float down = -bias * kLog2e;
      const uint32_t row = row0 + n;
      // keys that the row sees: those before this one
      const int64_t seen = row < rows ? base + token + 1 : 0;
      // whether some row of the tile is none, or must not see some key
      const bool masked = row0 + kRows > rows || row0 < ((int64_t)key0 + kKeys - 1 - base) * a.ratio;
      row0 += step;
      token += step_tokens;
      in_head += step_rest;
      if (in_head >= a.ratio) {
        in_head -= a.ratio;
        ++token;
      }
      if (row0 < rows) load();
      if (masked) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = __builtin_amdgcn_exp2f(fmaf(score[t][e], a.scale_log2, down));
            acc[t][e] += (int64_t)(key0 + 16 * t + 4 * g + e) < seen ? p : 0.f;
          }
      } else {
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[t][e] += __builtin_amdgcn_exp2f(fmaf(score[t][e], a.scale_log2, down));
      }
    }
    float mine = 0.f;
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = acc[t][e];
        x += turned<8>(x);
        x += turned<4>(x);
        x += turned<2>(x);
        x += turned<1>(x);
        if (n == 4 * t + e) mine = x;
      }
    if (split) {
      lds[wave][lane] = mine;
      __syncthreads();
      mine = lds[0][lane] + lds[1][lane] + (lds[2][lane] + lds[3][lane]);
      __syncthreads();
    }
    if (stored && !(split && wave > 0)) {
      a.weights_out[to] = sum + mine;
      if (is_new && a.born) a.born[to] = a.positions[seq.first + (uint32_t)(own - base)];
    }
  }
}

// Workgroups take units in turn, so that the first ones of a prompt, which most rows see, go out first and
// to different CUs. Each finds its own by walking over the sequences' lengths, 64 a step.
template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void weigh_kernel(WeighArgs a) {
  __shared__ float lds[kWaves][64];
  const uint32_t lane = threadIdx.x & 63;
  uint64_t before = 0;  // units of the sequences that were walked over
  uint64_t u = blockIdx.x;
  for (uint32_t s0 = 0; s0 < a.n_seq; s0 += 64) {
    Seq mine{};
    if (s0 + lane < a.n_seq) mine = seq_at<D>(a, s0 + lane);
    uint64_t upto = (uint64_t)mine.units * a.kv_heads;  // inclusive sum over the lanes
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint64_t x = __shfl_up(upto, d, 64);
      if ((int)lane >= d) upto += x;
    }
    const uint64_t all = __shfl(upto, 63, 64);
    for (; u < before + all; u += gridDim.x) {
      const uint32_t i = (uint32_t)__builtin_ctzll(__ballot(upto > u - before));
      Seq seq;
      seq.first = (uint32_t)__builtin_amdgcn_readlane((int)mine.first, (int)i);
      seq.tokens = (uint32_t)__builtin_amdgcn_readlane((int)mine.tokens, (int)i);
      seq.keys = (uint32_t)__builtin_amdgcn_readlane((int)mine.keys, (int)i);
      seq.units = (uint32_t)__builtin_amdgcn_readlane((int)mine.units, (int)i);
      const uint64_t end = __shfl(upto, (int)i, 64);
      const uint32_t in = uniform((uint32_t)(u - before - (end - (uint64_t)seq.units * a.kv_heads)));
      weigh_unit<T, D>(a, seq, s0 + i, in % a.kv_heads, in / a.kv_heads, lds);
    }
    before += all;
  }
}

template <class T>
void launch_weigh(const WeighArgs& a, uint32_t head_dim, uint32_t groups, hipStream_t s) {
  if (head_dim == 64) hipLaunchKernelGGL((weigh_kernel<T, 64>), dim3(groups), dim3(kThreads), 0, s, a);
  else if (head_dim == 128) hipLaunchKernelGGL((weigh_kernel<T, 128>), dim3(groups), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((weigh_kernel<T, 256>), dim3(groups), dim3(kThreads), 0, s, a);
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
  a.page_log2 = (uint32_t)log2_exact(kv->page_tokens);
  a.n_pages = (uint32_t)kv->n_pages;
  a.scale_log2 = in->scale * kLog2e;
  // no more than there are units of the smallest kind
  const uint64_t keys = in->own_width * kv->page_tokens;
  const uint64_t units = in->n_seq * kv->kv_heads * ((keys + 31) / 32);
  const uint32_t groups = (uint32_t)(units < kMostGroups ? units : kMostGroups);
  if (kv->dtype == GLEAM_FP16) launch_weigh<Fp16>(a, kv->head_dim, groups, (hipStream_t)stream);
  else launch_weigh<Bf16>(a, kv->head_dim, groups, (hipStream_t)stream);
  return launch_status("weigh_kernel");
}
