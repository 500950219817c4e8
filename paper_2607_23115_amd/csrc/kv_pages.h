// What the calls on a paged key/value cache share: the checks of its description, and
// 16-bit floating types on the device.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "gleam_internal.h"

namespace gleam {

// Sets the error text (with `who`) where kv is not a cache that the kernels can address.
gleam_status validate_kv(const gleam_kv_pages* kv, const char* who);
// Heads of a tensor [tokens, heads, head_dim]: pointer and strides that 16-byte loads can use.
gleam_status validate_heads(const void* p, const int64_t stride[2], const char* name, const char* who);

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2v __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4v __attribute__((ext_vector_type(4)));

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
