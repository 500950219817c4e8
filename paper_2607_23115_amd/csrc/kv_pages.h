// What the calls on a paged key/value cache share: the checks of its description, and
// 16-bit floating types on the device.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gleam_internal.h"

namespace gleam {

// Sets the error text (with `who`) where kv is not a cache that the kernels can address.
gleam_status validate_kv(const gleam_kv_pages* kv, const char* who);
// The same where places of keys, or of values, overlap: for calls that store into the cache.
gleam_status validate_places(const gleam_kv_pages* kv, const char* who);
// Bits of drafts: [n_tokens][words] of 64.
gleam_status validate_seen(const uint64_t* d_seen, uint32_t words, uint64_t n_tokens, const char* who);
// A ragged batch's sequences and the rows of their page table.
gleam_status validate_sequences(const gleam_kv_pages* kv, uint64_t n_seq, uint64_t own_width, const int32_t* d_own_pages,
                                const int32_t* d_own_len, const char* who);
// That the lengths a call returns overlap none of what its workgroups read at different times: they may have been
// written by then.
struct ReadLate {
  const void* p;
  uint64_t bytes;
  const char* name;
};
gleam_status validate_len_out(const int32_t* d_len_out, uint64_t n_seq, const ReadLate* reads, int n_reads,
                              const char* who);
// What is kept for each place and key head, 4 bytes in [n_pages][kv_heads][page_tokens], and where it goes.
gleam_status validate_tracked(const gleam_kv_pages* kv, const void* in, const void* out, const char* name,
                              const char* who);
// Heads of a tensor [tokens, heads, head_dim]: pointer and strides that 16-byte loads can use.
gleam_status validate_heads(const void* p, const int64_t stride[2], const char* name, const char* who);

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

constexpr uint64_t kMostSeq = 1ull << 20;  // sequences of a batch

struct Fp16 {
  typedef _Float16 scalar;
  typedef f16x8 vec8;
  // exponent bits of a 16-bit value: all set in infinities and NaN
  static constexpr uint32_t kExp = 0x7c00u;
};
struct Bf16 {
  typedef __bf16 scalar;
  typedef bf16x8 vec8;
  static constexpr uint32_t kExp = 0x7f80u;
};

}  // namespace gleam
