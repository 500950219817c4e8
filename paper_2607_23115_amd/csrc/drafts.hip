// Trees of drafted tokens: who sees whom, and what becomes of the keys of the path that was accepted.
// Both calls are a few loads long that wait for each other, and bound by those: a tree of 13 takes 1.8 us, 96 of
// up to 160 5.8 (three rounds of 64 drafts); the path of one sequence, 32 heads of 128, 3.4, those of 128, of up to
// 20 drafts and 8 heads of 256, 7.2 (6 MB read and written; 11.2 where each row's pages were looked up in turn).

#include "kv_device.h"
#include "launch_shape.h"

namespace gleam {

gleam_status validate_seen(const uint64_t* d_seen, uint32_t words, uint64_t n_tokens, const char* who) {
  if (words == 0) {
    set_error("%s: seen_words must not be 0", who);
    return GLEAM_E_INVALID;
  }
  if (words > 1u << 16) {
    set_error("%s: bits of more than 2^22 drafts", who);
    return GLEAM_E_UNSUPPORTED;
  }
  if (n_tokens > 0 && (!d_seen || (reinterpret_cast<uintptr_t>(d_seen) & 7))) {
    set_error("%s: seen must be non-null and 8-byte aligned", who);
    return GLEAM_E_INVALID;
  }
  return GLEAM_OK;
}

gleam_status validate_sequences(const gleam_kv_pages* kv, uint64_t n_seq, uint64_t own_width, const int32_t* d_own_pages,
                                const int32_t* d_own_len, const char* who) {
  if (n_seq > kMostSeq) {
    set_error("%s: more than 2^20 sequences", who);
    return GLEAM_E_UNSUPPORTED;
  }
  if (own_width > (uint64_t)INT32_MAX / kv->page_tokens) {
    set_error("%s: a table row of 2^31 keys or more", who);
    return GLEAM_E_INVALID;
  }
  if (n_seq > 0 && (!d_own_len || (own_width > 0 && !d_own_pages))) {
    set_error("%s: null own_len or own_pages", who);
    return GLEAM_E_INVALID;
  }
  return GLEAM_OK;
}

gleam_status validate_len_out(const int32_t* d_len_out, uint64_t n_seq, const ReadLate* reads, int n_reads,
                              const char* who) {
  const uintptr_t to = reinterpret_cast<uintptr_t>(d_len_out);
  for (int i = 0; i < n_reads; ++i) {
    const uintptr_t from = reinterpret_cast<uintptr_t>(reads[i].p);
    if (reads[i].bytes == 0) continue;
    if (from < to ? to - from < reads[i].bytes : from - to < 4 * n_seq) {
      set_error("%s: len_out must not overlap %s", who, reads[i].name);
      return GLEAM_E_INVALID;
    }
  }
  return GLEAM_OK;
}

namespace {

// --------------------------------------------------------------------------------------- //
// who sees whom
// --------------------------------------------------------------------------------------- //
struct TreeArgs {
  const int32_t* parent;
  const int32_t* q_first;
  uint64_t* seen;
  int32_t* depth;  // nullable
  uint32_t n_tokens, n_seq, words;
};

// A wave for each sequence takes its drafts 64 at a time, in order. Within the 64, each draft's pointer
// goes to its parent, then to its parent's pointer and so on: after six rounds of taking over the bits and
// the pointer of whom it points to, its bits hold the whole chain. What lies before the 64 is the row of
// the parent that the chain's first draft has there. The last workgroups clear tokens of no sequence.
__global__ __launch_bounds__(64) void tree_kernel(TreeArgs a) {
  const uint32_t lane = threadIdx.x;
  const int32_t all = (int32_t)a.n_tokens;
  const uint32_t before = a.n_seq ? (uint32_t)clamp_to(a.q_first[0], all) : 0;
  const uint32_t behind = a.n_seq ? (uint32_t)clamp_to(a.q_first[a.n_seq], all) : 0;
  if (blockIdx.x >= a.n_seq) {
    const uint32_t step = (gridDim.x - a.n_seq) * 64;
    for (uint64_t t = (blockIdx.x - a.n_seq) * 64 + lane; t < a.n_tokens; t += step) {
      if (t >= before && t < behind) continue;
      for (uint32_t w = 0; w < a.words; ++w) a.seen[t * a.words + w] = 0;
      if (a.depth) a.depth[t] = 0;
    }
    return;
  }
  uint32_t first = (uint32_t)clamp_to(a.q_first[blockIdx.x], all);
  uint32_t end = (uint32_t)clamp_to(a.q_first[blockIdx.x + 1], all);
  // of offsets that decrease, none that others clear
  first = first > before ? first : before;
  end = end < behind ? end : behind;
  if (end <= first) return;
  const uint32_t n = end - first;
  uint64_t* const seen = a.seen + (uint64_t)first * a.words;
  const int32_t* const parent = a.parent + first;
  int32_t* const depth = a.depth ? a.depth + first : nullptr;
  int32_t next = lane < n ? parent[lane] : -1;
  for (uint32_t from = 0; from < n; from += 64) {
    const uint32_t i = from + lane;
    int32_t p = next;
    next = i + 64 < n ? parent[i + 64] : -1;
    if (p < 0 || (uint32_t)p >= i) p = -1;  // no parent, or none that comes before it
    int32_t up = p >= (int32_t)from ? p - (int32_t)from : -1;
    uint64_t bits = 1ull << lane;
    int32_t count = 1;
#pragma unroll
    for (int round = 0; round < 6; ++round) {
      const int to = up < 0 ? (int)lane : up;
      const uint64_t their_bits = __shfl(bits, to, 64);
      const int32_t their_count = __shfl(count, to, 64), their_up = __shfl(up, to, 64);
      if (up >= 0) {
        bits |= their_bits;
        count += their_count;
        up = their_up;
      }
    }
    const int32_t out = __shfl(p, (int)__builtin_ctzll(bits), 64);  // an earlier 64's, or -1
    if (i < n) {
      for (uint32_t w = 0; w < a.words; ++w) {
        uint64_t x = 0;
        if (w == from / 64) x = bits;
        else if (w < from / 64 && out >= 0) x = seen[(uint64_t)out * a.words + w];
        seen[(uint64_t)i * a.words + w] = x;
      }
      if (depth) depth[i] = count - 1 + (out >= 0 ? depth[out] + 1 : 0);
    }
    __syncthreads();  // of one wave: what it has stored is read in later rounds
  }
}

// --------------------------------------------------------------------------------------- //
// the accepted path
// --------------------------------------------------------------------------------------- //
struct AcceptArgs {
  uint8_t* base[2];  // keys, values
  int64_t page[2], place[2], head[2];  // bytes
  const int32_t* q_first;
  const uint64_t* seen;
  const int32_t* leaf;
  const int32_t* own_pages;
  const int32_t* own_len;
  int32_t* len_out;
  uint32_t n_tokens, n_seq, words, own_width, page_log2, n_pages, kv_heads;
};

constexpr int kAcceptThreads = 256;
constexpr int kAcceptRows = 8;  // rows in flight

// The path's drafts, in order, are the leaf's bits. Draft number e of the path goes to where draft e was:
// never behind its own place, so a lane that takes 16 bytes of each row in turn overwrites none that it
// still has to read, and no other lane has to do with them. D / 8 lanes take a head's keys, others its
// values and the next heads. Where 64 drafts' keys are, and go to, is looked up at once, by a lane each.
template <int D>
__global__ __launch_bounds__(kAcceptThreads) void accept_kernel(AcceptArgs a) {
  constexpr uint32_t kLanes = D / 8;
  const uint32_t row = (blockIdx.y * kAcceptThreads + threadIdx.x) / kLanes;  // of keys, then of values
  const bool live = row < 2 * a.kv_heads;
  const int which = live && row >= a.kv_heads;
  uint8_t* const base = a.base[which] + (live ? row - which * a.kv_heads : 0) * a.head[which] +
                        threadIdx.x % kLanes * 16;
  const int64_t page_stride = a.page[which], place_stride = a.place[which];
  for (uint32_t s = blockIdx.x; s < a.n_seq; s += gridDim.x) {
    const uint32_t first = (uint32_t)clamp_to(a.q_first[s], (int32_t)a.n_tokens);
    const uint32_t end = (uint32_t)clamp_to(a.q_first[s + 1], (int32_t)a.n_tokens);
    const uint32_t n = end > first ? end - first : 0;
    const int32_t leaf = a.leaf[s];
    const uint32_t own = a.n_pages ? (uint32_t)clamp_to(a.own_len[s], (int32_t)(a.own_width << a.page_log2)) : 0;
    const int64_t draft = (int64_t)own - n;  // the first draft's key
    const uint32_t kept = draft < 0 ? 0 : (uint32_t)draft;  // the keys before
    uint32_t path = 0;
    if (leaf >= 0 && (uint32_t)leaf < n) {
      const uint64_t* const bits = a.seen + (uint64_t)(first + leaf) * a.words;
      const int32_t* const pages = a.own_pages + (uint64_t)s * a.own_width;
      const uint32_t lane = threadIdx.x & 63, mask = (1u << a.page_log2) - 1;
      for (uint32_t word = 0; word < a.words && word * 64 < n; ++word) {
        const uint32_t j = word * 64 + lane;
        const int64_t key = draft + j;
        const uint64_t on = __ballot((bits[word] >> lane & 1) && j < n && key >= 0);
        const uint32_t src = (uint32_t)key, dst = kept + path + (uint32_t)__popcll(on & ((1ull << lane) - 1));
        path += (uint32_t)__popcll(on);
        uint32_t src_page = kNoPage, dst_page = kNoPage;
        if ((on >> lane & 1) && src != dst) {
          src_page = (uint32_t)pages[src >> a.page_log2];
          dst_page = (uint32_t)pages[dst >> a.page_log2];
        }
        uint64_t todo = __ballot(src_page < a.n_pages && dst_page < a.n_pages);
        while (todo) {
          u32x4v data[kAcceptRows];
          int64_t to[kAcceptRows];
#pragma unroll
          for (int r = 0; r < kAcceptRows; ++r) {
            to[r] = -1;
            if (!todo) continue;
            const int at = __builtin_ctzll(todo);
            todo &= todo - 1;
            auto get = [at](uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, at); };
            const uint8_t* const from = base + (int64_t)get(src_page) * page_stride + (int64_t)(get(src) & mask) * place_stride;
            to[r] = (int64_t)get(dst_page) * page_stride + (int64_t)(get(dst) & mask) * place_stride;
            if (live) data[r] = *reinterpret_cast<const u32x4v*>(from);
          }
#pragma unroll
          for (int r = 0; r < kAcceptRows; ++r)
            if (live && to[r] >= 0) *reinterpret_cast<u32x4v*>(base + to[r]) = data[r];
        }
      }
    }
    if (blockIdx.y == 0 && threadIdx.x == 0) a.len_out[s] = (int32_t)(kept + path);
  }
}

}  // namespace

hipError_t preload_drafts() {
  hipFuncAttributes attr;
  return hipFuncGetAttributes(&attr, reinterpret_cast<const void*>(&tree_kernel));
}

}  // namespace gleam

extern "C" gleam_status gleam_draft_tree(const int32_t* d_parent, const int32_t* d_q_first, uint64_t n_tokens,
                                         uint64_t n_seq, uint64_t* d_seen, uint32_t seen_words, int32_t* d_depth,
                                         void* stream) {
  using namespace gleam;
  clear_error();
  const char* const who = "gleam_draft_tree";
  gleam_status st = validate_seen(d_seen, seen_words, n_tokens, who);
  if (st != GLEAM_OK) return st;
  if (n_seq > kMostSeq || n_tokens > INT32_MAX) {
    set_error("%s: more than 2^20 sequences, or 2^31 tokens", who);
    return GLEAM_E_UNSUPPORTED;
  }
  if (n_tokens == 0) return GLEAM_OK;
  if (!d_parent || (n_seq > 0 && !d_q_first)) {
    set_error("%s: null parent or q_first", who);
    return GLEAM_E_INVALID;
  }
  const TreeArgs a{d_parent, d_q_first, d_seen, d_depth, (uint32_t)n_tokens, (uint32_t)n_seq, seen_words};
  // those that clear take four rounds each, up to a workgroup a CU
  const uint64_t clear = (n_tokens + 255) / 256;
  hipLaunchKernelGGL(tree_kernel, dim3((uint32_t)(n_seq + (clear < 256 ? clear : 256))), dim3(64), 0,
                     (hipStream_t)stream, a);
  return launch_status("tree_kernel");
}

extern "C" gleam_status gleam_kv_accept(const gleam_kv_pages* kv, const gleam_accept* in, void* stream) {
  using namespace gleam;
  clear_error();
  const char* const who = "gleam_kv_accept";
  gleam_status st = validate_kv(kv, who);
  if (st != GLEAM_OK) return st;
  if (!in) {
    set_error("%s: null arguments", who);
    return GLEAM_E_INVALID;
  }
  if ((st = validate_seen(in->d_seen, in->seen_words, in->n_tokens, who)) != GLEAM_OK) return st;
  if ((st = validate_sequences(kv, in->n_seq, in->own_width, in->d_own_pages, in->d_own_len, who)) != GLEAM_OK)
    return st;
  if ((st = validate_places(kv, who)) != GLEAM_OK) return st;
  if (in->n_tokens > INT32_MAX) {
    set_error("%s: 2^31 tokens or more", who);
    return GLEAM_E_UNSUPPORTED;
  }
  if (in->n_seq == 0) return GLEAM_OK;
  if (!in->d_q_first || !in->d_leaf || !in->d_len_out) {
    set_error("%s: null q_first, leaf or len_out", who);
    return GLEAM_E_INVALID;
  }
  const ReadLate reads[] = {{in->d_own_len, 4 * in->n_seq, "own_len"},
                            {in->d_leaf, 4 * in->n_seq, "leaf"},
                            {in->d_q_first, 4 * (in->n_seq + 1), "q_first"},
                            {in->d_seen, 8 * in->n_tokens * in->seen_words, "seen"},
                            {in->d_own_pages, 4 * in->n_seq * in->own_width, "own_pages"}};
  if ((st = validate_len_out(in->d_len_out, in->n_seq, reads, 5, who)) != GLEAM_OK) return st;
  AcceptArgs a{};
  a.base[0] = static_cast<uint8_t*>(kv->d_k);
  a.base[1] = static_cast<uint8_t*>(kv->d_v);
  const int64_t* const stride[2] = {kv->k_stride, kv->v_stride};
  for (int i = 0; i < 2; ++i) {
    a.page[i] = 2 * stride[i][0];
    a.place[i] = 2 * stride[i][1];
    a.head[i] = 2 * stride[i][2];
  }
  a.q_first = in->d_q_first;
  a.seen = in->d_seen;
  a.leaf = in->d_leaf;
  a.own_pages = in->d_own_pages;
  a.own_len = in->d_own_len;
  a.len_out = in->d_len_out;
  a.n_tokens = (uint32_t)in->n_tokens;
  a.n_seq = (uint32_t)in->n_seq;
  a.words = in->seen_words;
  a.own_width = (uint32_t)in->own_width;
  a.page_log2 = (uint32_t)log2_exact(kv->page_tokens);
  a.n_pages = (uint32_t)kv->n_pages;
  a.kv_heads = kv->kv_heads;
  const uint32_t y = (2 * kv->kv_heads * (kv->head_dim / 8) + kAcceptThreads - 1) / kAcceptThreads;
  const uint64_t most = max_workgroups(kAcceptThreads) / y;
  const dim3 grid((uint32_t)(in->n_seq < most ? in->n_seq : most), y);
  hipStream_t s = (hipStream_t)stream;
  if (kv->head_dim == 64) hipLaunchKernelGGL(accept_kernel<64>, grid, dim3(kAcceptThreads), 0, s, a);
  else if (kv->head_dim == 128) hipLaunchKernelGGL(accept_kernel<128>, grid, dim3(kAcceptThreads), 0, s, a);
  else hipLaunchKernelGGL(accept_kernel<256>, grid, dim3(kAcceptThreads), 0, s, a);
  return launch_status("accept_kernel");
}
