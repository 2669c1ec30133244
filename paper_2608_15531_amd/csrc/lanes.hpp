// Reductions over the lanes of a wave by data-parallel moves and lane swaps, without LDS.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fqk {

// v of another lane of the same 16: quad_perm, mirror and half-mirror controls of DPP.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  const int x = __builtin_bit_cast(int, v);
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(x, x, CTRL, 0xF, 0xF, true));
}

// f(v of this lane, v of lane ^ 16) and the same for lane ^ 32, in the lanes' order on
// both sides: the result is the same in both lanes.
template <class F>
__device__ __forceinline__ float across16(float v, F f) {
  const uint32_t x = __builtin_bit_cast(uint32_t, v);
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  return f(__builtin_bit_cast(float, uint32_t(r[0])), __builtin_bit_cast(float, uint32_t(r[1])));
}
template <class F>
__device__ __forceinline__ float across32(float v, F f) {
  const uint32_t x = __builtin_bit_cast(uint32_t, v);
  const auto r = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return f(__builtin_bit_cast(float, uint32_t(r[0])), __builtin_bit_cast(float, uint32_t(r[1])));
}

struct Max {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Min {
  __device__ __forceinline__ float operator()(float a, float b) const { return fminf(a, b); }
};
struct Add {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};

// Over each N = 8, 16 or 64 neighbouring lanes, the result in all of them.
template <int N, class F>
__device__ __forceinline__ float over_lanes(float v, F f) {
  static_assert(N == 8 || N == 16 || N == 64, "lanes");
  v = f(v, dpp<0xB1>(v));                     // quad_perm 1 0 3 2
  v = f(v, dpp<0x4E>(v));                     // quad_perm 2 3 0 1
  v = f(v, dpp<0x141>(v));                    // half mirror: the other four of eight
  if constexpr (N >= 16) v = f(v, dpp<0x140>(v));   // mirror: the other eight of sixteen
  if constexpr (N == 64) {
    v = across16(v, f);
    v = across32(v, f);
  }
  return v;
}

}  // namespace fqk
