// Appending to a paged key/value cache: each token's keys are normed (where the model norms its
// heads), rotated by the token's position and stored with its values in the token's place of a
// page; the token's queries are normed and rotated in the same pass.
//
// With c, s the cosine and sine of position * f_i, a pair (a, b) of a head's dimensions becomes
// (a c - b s, b c + a s). Pairs are (i, i + r/2) or (2i, 2i + 1) of the first r dimensions.
//
// Every value is read once and written once, with some ten operations between: bound by memory
// for many tokens, by the time of one load and one store for few. head_dim / 16 lanes take a
// head, 16 dimensions each, so that both members of 8 pairs are in one lane (no exchange for the
// rotation; the norm's sum takes log2(head_dim / 16) exchanges) and every access is 16 bytes. A
// lane rotates the same pairs of every head, so a wave that keeps to one token loads its cosines
// and sines once. 16,384 tokens of 32 and 8 heads of 128: 84 us, 4.9 TB/s (a copy of as many bytes
// 78 us); one token 2.6 us.

#include <algorithm>

#include "kv_pages.h"
#include "launch_shape.h"

namespace gleam {

gleam_status validate_heads(const void* p, const int64_t stride[2], const char* name, const char* who) {
  if (!p || (reinterpret_cast<uintptr_t>(p) & 15)) {
    set_error("%s: %s must be non-null and 16-byte aligned", who, name);
    return GLEAM_E_INVALID;
  }
  if ((stride[0] & 7) || (stride[1] & 7) || stride[0] < 0 || stride[1] < 0) {
    set_error("%s: strides of %s must be multiples of 8 elements", who, name);
    return GLEAM_E_INVALID;
  }
  return GLEAM_OK;
}

gleam_status validate_kv(const gleam_kv_pages* kv, const char* who) {
  if (!kv) {
    set_error("%s: null cache", who);
    return GLEAM_E_INVALID;
  }
  if (kv->dtype != GLEAM_FP16 && kv->dtype != GLEAM_BF16) {
    set_error("%s: dtype must be GLEAM_FP16 or GLEAM_BF16", who);
    return GLEAM_E_INVALID;
  }
  if (kv->head_dim != 64 && kv->head_dim != 128 && kv->head_dim != 256) {
    set_error("%s: head_dim must be 64, 128 or 256", who);
    return GLEAM_E_INVALID;
  }
  if (kv->kv_heads < 1 || kv->kv_heads > 65535) {
    set_error("%s: kv_heads must be 1 to 65535", who);
    return GLEAM_E_INVALID;
  }
  const int page_log2 = log2_exact(kv->page_tokens);
  if (page_log2 < 4 || page_log2 > 12) {
    set_error("%s: page_tokens must be a power of two from 16 to 4096", who);
    return GLEAM_E_INVALID;
  }
  if (kv->n_pages > INT32_MAX) {
    set_error("%s: more than 2^31 - 1 pages", who);
    return GLEAM_E_INVALID;
  }
  const void* const p[2] = {kv->d_k, kv->d_v};
  const int64_t* const stride[2] = {kv->k_stride, kv->v_stride};
  for (int i = 0; i < 2; ++i) {
    if (kv->n_pages > 0 && (!p[i] || (reinterpret_cast<uintptr_t>(p[i]) & 15))) {
      set_error("%s: keys and values must be non-null and 16-byte aligned", who);
      return GLEAM_E_INVALID;
    }
    for (int j = 0; j < 3; ++j) {
      if (stride[i][j] < 0 || (stride[i][j] & 7)) {
        set_error("%s: strides of keys and values must be multiples of 8 elements", who);
        return GLEAM_E_INVALID;
      }
    }
  }
  return GLEAM_OK;
}

namespace {

// Whether no element belongs to two places: each stride is at least what the smaller ones span.
// (Places that interleave without meeting, of strides that none of the usual orders has, are not
// told from those that overlap.)
bool places_apart(const gleam_kv_pages& kv, const int64_t stride[3]) {
  struct Dim {
    int64_t stride;
    uint64_t count;
  } dim[3] = {{stride[0], kv.n_pages}, {stride[1], kv.page_tokens}, {stride[2], kv.kv_heads}};
  std::sort(dim, dim + 3, [](const Dim& a, const Dim& b) { return a.stride < b.stride; });
  unsigned __int128 span = kv.head_dim;
  for (const Dim& d : dim) {
    if (d.count < 2) continue;
    if ((uint64_t)d.stride < span) return false;
    span += (unsigned __int128)d.stride * (d.count - 1);
  }
  return true;
}

}  // namespace

gleam_status validate_places(const gleam_kv_pages* kv, const char* who) {
  // a place that two heads or two tokens share would take whichever is stored last
  if (!places_apart(*kv, kv->k_stride) || !places_apart(*kv, kv->v_stride)) {
    set_error("%s: pages, places and heads of the cache overlap", who);
    return GLEAM_E_INVALID;
  }
  return GLEAM_OK;
}

namespace {

constexpr int kAppendThreads = 256, kAppendWaves = kAppendThreads / 64;

struct AppendArgs {
  const uint8_t* src[3];  // queries, keys, values
  uint8_t* dst[3];
  int64_t src_token[3], src_head[3];  // strides in bytes
  int64_t dst_page[2], dst_place[2], dst_head[2];  // keys, values
  const uint8_t* weight[2];
  const float* rotary;
  const int64_t* slots;
  const int32_t* positions;
  uint64_t n_tokens, n_slots, rotary_positions;
  uint32_t q_heads, kv_heads, rot_dim, page_log2;
  uint32_t splits;  // waves per token
  float eps;
};

template <class T, int D, bool kInterleaved>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(AppendArgs a) {
  typedef typename T::vec8 vec8;
  typedef typename T::scalar scalar;
  constexpr uint32_t kLanes = D / 16, kRows = 64 / kLanes;  // lanes per head, heads per wave and round
  const uint64_t wave = (uint64_t)blockIdx.x * kAppendWaves + (threadIdx.x >> 6);
  const uint64_t token = wave / a.splits;
  if (token >= a.n_tokens) return;
  const uint32_t split = (uint32_t)(wave - token * a.splits);
  const uint32_t lane = threadIdx.x & 63, p = lane % kLanes, sub = lane / kLanes;

  const uint64_t slot = (uint64_t)a.slots[token];
  const bool stored = slot < a.n_slots;
  const uint64_t page = slot >> a.page_log2, place = slot & ((1u << a.page_log2) - 1);

  // the lane's two runs of 8 dimensions
  const uint32_t half8 = a.rot_dim / 16;
  const bool rotates = p < half8;
  uint32_t c0 = 2 * p, c1 = 2 * p + 1;
  if (!kInterleaved && rotates) {
    c0 = p;
    c1 = p + half8;
  }
  f32x4 cs[2], sn[2];
  if (rotates) {
    const int64_t pos = a.positions[token];
    if (pos >= 0 && (uint64_t)pos < a.rotary_positions) {
      const float* row = a.rotary + (uint64_t)pos * a.rot_dim + 8 * p;
      cs[0] = *reinterpret_cast<const f32x4*>(row);
      cs[1] = *reinterpret_cast<const f32x4*>(row + 4);
      sn[0] = *reinterpret_cast<const f32x4*>(row + 8 * half8);
      sn[1] = *reinterpret_cast<const f32x4*>(row + 8 * half8 + 4);
    } else {
      cs[0] = cs[1] = sn[0] = sn[1] = (f32x4)__builtin_nanf("");
    }
  }

  const uint32_t rows = a.q_heads + 2 * a.kv_heads;
  for (uint32_t r0 = split * kRows; r0 < rows; r0 += a.splits * kRows) {
    const uint32_t r = r0 + sub;
    const uint32_t part = r < a.q_heads ? 0 : r < a.q_heads + a.kv_heads ? 1 : 2;
    const uint32_t head = part == 0 ? r : part == 1 ? r - a.q_heads : r - a.q_heads - a.kv_heads;
    const bool live = r < rows && (part == 0 || stored);
    vec8 v0{}, v1{};
    if (live) {
      const uint8_t* src = (part == 0 ? a.src[0] : part == 1 ? a.src[1] : a.src[2]) +
                           (int64_t)token * (part == 0 ? a.src_token[0] : part == 1 ? a.src_token[1] : a.src_token[2]) +
                           (int64_t)head * (part == 0 ? a.src_head[0] : part == 1 ? a.src_head[1] : a.src_head[2]);
      v0 = *reinterpret_cast<const vec8*>(src + 16 * c0);
      v1 = *reinterpret_cast<const vec8*>(src + 16 * c1);
    }
    float x[16];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = (float)v0[i];
      x[8 + i] = (float)v1[i];
    }
    if (a.weight[0] || a.weight[1]) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) sum += x[i] * x[i];
#pragma unroll
      for (uint32_t o = 1; o < kLanes; o <<= 1) sum += __shfl_xor(sum, (int)o, 64);
      const uint8_t* w = part == 0 ? a.weight[0] : part == 1 ? a.weight[1] : nullptr;
      if (w) {
        const float scale = 1.0f / sqrtf(sum * (1.0f / D) + a.eps);
        const vec8 w0 = *reinterpret_cast<const vec8*>(w + 16 * c0);
        const vec8 w1 = *reinterpret_cast<const vec8*>(w + 16 * c1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = x[i] * scale * (float)w0[i];
          x[8 + i] = x[8 + i] * scale * (float)w1[i];
        }
      }
    }
    if (rotates && part != 2) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float c = cs[i >> 2][i & 3], s = sn[i >> 2][i & 3];
        const int ia = kInterleaved ? 2 * i : i, ib = kInterleaved ? 2 * i + 1 : 8 + i;
        const float u = x[ia], v = x[ib];
        x[ia] = u * c - v * s;
        x[ib] = v * c + u * s;
      }
    }
    if (live) {
      uint8_t* dst;
      if (part == 0) {
        dst = a.dst[0] + (token * a.q_heads + head) * (uint64_t)(2 * D);
      } else {
        const int i = part == 2;
        dst = (i ? a.dst[2] : a.dst[1]) + (int64_t)page * (i ? a.dst_page[1] : a.dst_page[0]) +
              (int64_t)place * (i ? a.dst_place[1] : a.dst_place[0]) +
              (int64_t)head * (i ? a.dst_head[1] : a.dst_head[0]);
      }
      if (part != 2) {  // values are stored bit for bit
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          v0[i] = (scalar)x[i];
          v1[i] = (scalar)x[8 + i];
        }
      }
      *reinterpret_cast<vec8*>(dst + 16 * c0) = v0;
      *reinterpret_cast<vec8*>(dst + 16 * c1) = v1;
    }
  }
}

template <class T, int D>
void launch_append(const AppendArgs& a, bool interleaved, uint32_t groups, hipStream_t stream) {
  if (interleaved)
    hipLaunchKernelGGL((append_kernel<T, D, true>), dim3(groups), dim3(kAppendThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((append_kernel<T, D, false>), dim3(groups), dim3(kAppendThreads), 0, stream, a);
}

// One thread per angle: a power, a product and a sine and cosine in 64 bits. A table is made
// once, so nothing here is tuned.
__global__ __launch_bounds__(256) void rotary_table_kernel(float* table, uint64_t positions, uint32_t half, double base,
                                                           double factor, double original, double slow, double fast,
                                                           double magnitude) {
  const uint32_t i = blockIdx.y * 256 + threadIdx.x;
  if (i >= half) return;
  double f = pow(base, -(double)(2 * i) / (double)(2 * half));
  double keep = 0.0;
  if (original > 0.0) {
    keep = (original * f * 0.15915494309189533577 - slow) / (fast - slow);
    keep = fmin(fmax(keep, 0.0), 1.0);
  }
  f *= keep + (1.0 - keep) / factor;
  for (uint64_t p = blockIdx.x; p < positions; p += gridDim.x) {
    double s, c;
    sincos((double)p * f, &s, &c);
    float* row = table + p * (2 * half);
    row[i] = (float)(c * magnitude);
    row[half + i] = (float)(s * magnitude);
  }
}

}  // namespace

hipError_t preload_kv_append() {
  hipFuncAttributes attr;
  return hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&append_kernel<Bf16, 128, false>));
}

}  // namespace gleam

extern "C" gleam_status gleam_rotary_table(float* d_table, uint64_t positions, uint32_t rot_dim, double base,
                                           double factor, double original_positions, double slow, double fast,
                                           double magnitude, void* stream) {
  using namespace gleam;
  clear_error();
  if (rot_dim == 0 || (rot_dim & 1) || rot_dim > 65536 || positions > INT32_MAX) {
    set_error("gleam_rotary_table: rot_dim must be even, 2 to 65536, and positions below 2^31");
    return GLEAM_E_INVALID;
  }
  // written so that a NaN is refused too
  if (!(base > 0.0 && factor > 0.0 && original_positions >= 0.0 && fast > slow)) {
    set_error("gleam_rotary_table: base and factor must be positive, original_positions not negative, fast above slow");
    return GLEAM_E_INVALID;
  }
  if (positions == 0) return GLEAM_OK;
  if (!d_table) {
    set_error("gleam_rotary_table: null table");
    return GLEAM_E_INVALID;
  }
  const uint32_t x = (uint32_t)(positions < 4096 ? positions : 4096);
  hipLaunchKernelGGL(rotary_table_kernel, dim3(x, (rot_dim / 2 + 255) / 256), dim3(256), 0, (hipStream_t)stream,
                     d_table, positions, rot_dim / 2, base, factor, original_positions, slow, fast, magnitude);
  return launch_status("rotary_table_kernel");
}

extern "C" gleam_status gleam_kv_append(const gleam_kv_pages* kv, const gleam_append* in, void* stream) {
  using namespace gleam;
  clear_error();
  const char* const who = "gleam_kv_append";
  gleam_status st = validate_kv(kv, who);
  if (st != GLEAM_OK) return st;
  if (!in) {
    set_error("%s: null arguments", who);
    return GLEAM_E_INVALID;
  }
  if (in->n_tokens == 0) return GLEAM_OK;
  if ((st = validate_heads(in->d_k, in->k_stride, "k", who)) != GLEAM_OK) return st;
  if ((st = validate_heads(in->d_v, in->v_stride, "v", who)) != GLEAM_OK) return st;
  if (!in->d_q != !in->d_q_out || (!in->d_q && in->q_heads != 0) || (in->d_q && in->q_heads == 0)) {
    set_error("%s: queries need d_q, d_q_out and q_heads together", who);
    return GLEAM_E_INVALID;
  }
  if (in->d_q) {
    const int64_t whole[2] = {0, 0};
    if ((st = validate_heads(in->d_q, in->q_stride, "q", who)) != GLEAM_OK) return st;
    if ((st = validate_heads(in->d_q_out, whole, "q_out", who)) != GLEAM_OK) return st;
  }
  if (in->q_heads > 65535) {
    set_error("%s: more than 65535 query heads", who);
    return GLEAM_E_INVALID;
  }
  const void* const weights[2] = {in->d_q_weight, in->d_k_weight};
  for (const void* w : weights) {
    if (reinterpret_cast<uintptr_t>(w) & 15) {
      set_error("%s: weights must be 16-byte aligned", who);
      return GLEAM_E_INVALID;
    }
  }
  if (in->d_rotary && (in->rot_dim == 0 || (in->rot_dim & 15) || in->rot_dim > kv->head_dim || !in->d_positions ||
                       (reinterpret_cast<uintptr_t>(in->d_rotary) & 15))) {
    set_error("%s: a rotary table needs positions, 16-byte alignment and a rot_dim that is a multiple of 16 up to "
              "head_dim", who);
    return GLEAM_E_INVALID;
  }
  if (!in->d_slots) {
    set_error("%s: null slots", who);
    return GLEAM_E_INVALID;
  }
  const int64_t* const strides[2] = {kv->k_stride, kv->v_stride};
  if ((st = validate_places(kv, who)) != GLEAM_OK) return st;
  if (in->n_tokens > INT32_MAX) {
    set_error("%s: 2^31 tokens or more", who);
    return GLEAM_E_UNSUPPORTED;
  }
  AppendArgs a{};
  a.src[0] = static_cast<const uint8_t*>(in->d_q);
  a.src[1] = static_cast<const uint8_t*>(in->d_k);
  a.src[2] = static_cast<const uint8_t*>(in->d_v);
  const int64_t* const src_stride[3] = {in->q_stride, in->k_stride, in->v_stride};
  for (int i = 0; i < 3; ++i) {
    a.src_token[i] = 2 * src_stride[i][0];
    a.src_head[i] = 2 * src_stride[i][1];
  }
  a.dst[0] = static_cast<uint8_t*>(in->d_q_out);
  a.dst[1] = static_cast<uint8_t*>(kv->d_k);
  a.dst[2] = static_cast<uint8_t*>(kv->d_v);
  for (int i = 0; i < 2; ++i) {
    a.dst_page[i] = 2 * strides[i][0];
    a.dst_place[i] = 2 * strides[i][1];
    a.dst_head[i] = 2 * strides[i][2];
    a.weight[i] = static_cast<const uint8_t*>(weights[i]);
  }
  a.rotary = in->d_rotary;
  a.slots = in->d_slots;
  a.positions = in->d_positions;
  a.n_tokens = in->n_tokens;
  a.page_log2 = (uint32_t)log2_exact(kv->page_tokens);
  a.n_slots = kv->n_pages << a.page_log2;
  a.rotary_positions = in->rotary_positions;
  a.q_heads = in->q_heads;
  a.kv_heads = kv->kv_heads;
  a.rot_dim = in->d_rotary ? in->rot_dim : 0;
  a.eps = in->eps;
  // A wave that keeps to one token loads its cosines and sines once; with few tokens there are
  // fewer such waves than the GPU holds (256 CUs of 32), and heads go to waves of their own.
  const uint32_t per_round = 64 / (kv->head_dim / 16);
  const uint32_t rounds = (in->q_heads + 2 * kv->kv_heads + per_round - 1) / per_round;
  const uint64_t want = (8192 + in->n_tokens - 1) / in->n_tokens;
  a.splits = (uint32_t)(want < rounds ? want : rounds);
  const uint64_t groups = (in->n_tokens * a.splits + kAppendWaves - 1) / kAppendWaves;
  if (groups > max_workgroups(kAppendThreads)) {
    set_error("%s: more tokens than one launch holds", who);
    return GLEAM_E_UNSUPPORTED;
  }
  const bool il = in->interleaved != 0;
  hipStream_t s = (hipStream_t)stream;
  const uint32_t n = (uint32_t)groups;
  if (kv->dtype == GLEAM_FP16) {
    kv->head_dim == 64    ? launch_append<Fp16, 64>(a, il, n, s)
    : kv->head_dim == 128 ? launch_append<Fp16, 128>(a, il, n, s)
                          : launch_append<Fp16, 256>(a, il, n, s);
  } else {
    kv->head_dim == 64    ? launch_append<Bf16, 64>(a, il, n, s)
    : kv->head_dim == 128 ? launch_append<Bf16, 128>(a, il, n, s)
                          : launch_append<Bf16, 256>(a, il, n, s);
  }
  return launch_status("append_kernel");
}
