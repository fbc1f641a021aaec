// Rotary positions: the table of cosines and sines, and the rotation of a
// row's channels on its way.
#pragma once

#include "ptc_kv.cuh"

namespace ptc {

template <typename T>
struct Half16;
template <>
struct Half16<__nv_bfloat16> {
  using Two = __nv_bfloat162;
  static constexpr bool kBf16 = true;
  static __device__ __forceinline__ float get(__nv_bfloat16 x) { return __bfloat162float(x); }
  static __device__ __forceinline__ __nv_bfloat16 put(float x) { return __float2bfloat16_rn(x); }
  static __device__ __forceinline__ __nv_bfloat16 put(double x) { return __double2bfloat16(x); }
  static __device__ __forceinline__ float2 get2(uint32_t x) {
    return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u));
  }
  // Whether 32 bits that are within 2 units in their last place may lie on the
  // other side of a rounding's border, or are too small for such a bound.
  static __device__ __forceinline__ bool unsure(float x) {
    const uint32_t u = __float_as_uint(x);
    return ((u & 0xFFFFu) - 0x7FFEu <= 4u) | (fabsf(x) < 0x1p-90f && x != 0.f);
  }
};
template <>
struct Half16<__half> {
  using Two = __half2;
  static constexpr bool kBf16 = false;
  static __device__ __forceinline__ float get(__half x) { return __half2float(x); }
  static __device__ __forceinline__ __half put(float x) { return __float2half_rn(x); }
  static __device__ __forceinline__ __half put(double x) { return __double2half(x); }
  static __device__ __forceinline__ float2 get2(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }
  // (among fp16's subnormals the border lies elsewhere)
  static __device__ __forceinline__ bool unsure(float x) {
    const uint32_t u = __float_as_uint(x);
    return ((u & 0x1FFFu) - 0xFFEu <= 4u) | (fabsf(x) < 0x1p-13f && x != 0.f);
  }
};

template <typename T>
__device__ __forceinline__ uint32_t bits16(T x) {
  return *reinterpret_cast<const uint16_t*>(&x);
}

// x c - y s of 16-bit x and y, rounded once: 32 bits give it to one unit in
// their last place (the rounding of y s is added back), and where that may lie
// on the other side of a border (or is not finite: what is left of an infinite
// product is NaN), 64 bits hold both products.  So a quantised
// cache's codes do not hang on how an angle's product was rounded.
template <typename T>
__device__ __noinline__ uint32_t turn_wide(float x, float c, float y, float s) {
  return bits16(Half16<T>::put((double)x * (double)c - (double)y * (double)s));
}
template <typename T>
__device__ __forceinline__ uint32_t turn(float x, float c, float y, float s) {
  const float p = y * s, e = fmaf(y, s, -p);
  const float z = fmaf(x, c, -p) - e;
  if (Half16<T>::unsure(z) || !(fabsf(z) < INFINITY)) return turn_wide<T>(x, c, y, s);
  return bits16(Half16<T>::put(z));
}

// How new tokens are turned.  pos: their positions, or null where a token's
// position is its place in its context.
struct RopeView {
  const float* table;
  const uint32_t* pos;
  uint32_t n_pos, n_freq;
  bool interleaved;
};

// The host-side checks of a ptc_rope, and its device view.
inline ptc_status rope_view(const ptc_rope* rope, uint32_t head_dim, RopeView* o) {
  if (rope->n_freq < 1 || rope->n_freq > head_dim / 2 || (rope->n_pos && !rope->table)) return PTC_ERR_INVALID_ARG;
  if ((uintptr_t)rope->table & 15) return PTC_ERR_INVALID_ARG;
  if (rope->interleaved != 0 && rope->interleaved != 1) return PTC_ERR_INVALID_ARG;
  o->table = rope->table;
  o->pos = rope->pos;
  o->n_pos = rope->n_pos;
  o->n_freq = rope->n_freq;
  o->interleaved = rope->interleaved != 0;
  return PTC_OK;
}

}  // namespace ptc
