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

// Memory behind an address that is the same in all lanes, or none: loads from none give 0 and go nowhere, so that
// a loop can ask for what it may not need without a branch.
typedef __amdgpu_buffer_rsrc_t Window;
__device__ inline Window window(const uint8_t* base, bool there) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), 0, (int)uniform(there ? ~0u : 0u), 0x00020000);
}
// 4, 8 or 16 bytes at the lane's offset and one that is the same in all lanes; kOnce: what nobody reads again
// soon is not kept in the caches.
template <class V, bool kOnce>
__device__ inline V load_from(Window w, uint32_t lane_offset, uint32_t offset) {
  constexpr int kPolicy = kOnce ? 2 : 0;
  if constexpr (sizeof(V) == 16) return __builtin_amdgcn_raw_buffer_load_b128(w, (int)lane_offset, (int)offset, kPolicy);
  else if constexpr (sizeof(V) == 8) return __builtin_amdgcn_raw_buffer_load_b64(w, (int)lane_offset, (int)offset, kPolicy);
  else return __builtin_amdgcn_raw_buffer_load_b32(w, (int)lane_offset, (int)offset, kPolicy);
}

// Waits for a value here. Where a branch may have asked for it, whatever uses it behind the branch would wait for
// all loads, those on their way for later among them.
template <class V>
__device__ inline void arrived(V& x) {
  asm volatile("" : "+v"(x));
}

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
