// Device code that the calls on a paged key/value cache share.
#pragma once

#include "kv_pages.h"

namespace gleam {

constexpr float kLog2e = 1.44269504088896340736f;

__device__ inline int32_t clamp_to(int32_t v, int32_t most) { return v < 0 ? 0 : v > most ? most : v; }

// Of a value that is the same in all lanes: kept in a scalar register, branches on it not masked.
__device__ inline uint32_t uniform(uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); }

// A number that no cache has a page of.
constexpr uint32_t kNoPage = ~0u;

// Products of 16 x 32 by 32 x 16 values.
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

}  // namespace gleam
