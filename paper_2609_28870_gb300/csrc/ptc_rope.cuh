// Rotary positions: the table of cosines and sines, and the rotation of a
// row's channels on its way.
#pragma once

#include "ptc_kv.cuh"
#include "ptc_tc.cuh"

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
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  static constexpr float kExact = 0x1p-15f;  // sums of numbers whose sizes are no further apart are exact in 32 bits
  // Whether 32 bits that are within 4 units in their last place may lie on the
  // other side of a rounding's border, or are too small for such a bound.
  static __device__ __forceinline__ bool unsure(float x) {
    const uint32_t u = __float_as_uint(x);
    return ((u & 0xFFFFu) - 0x7FFCu <= 8u) | (fabsf(x) < 0x1p-90f && x != 0.f);
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
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 x = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  static constexpr float kExact = 0x1p-12f;
  // (among fp16's subnormals the border lies elsewhere)
  static __device__ __forceinline__ bool unsure(float x) {
    const uint32_t u = __float_as_uint(x);
    return ((u & 0x1FFFu) - 0xFFCu <= 8u) | (fabsf(x) < 0x1p-13f && x != 0.f);
  }
};

template <typename Two>
__device__ __forceinline__ uint32_t fma_bits(uint32_t a, uint32_t b, uint32_t c) {
  const Two d = __hfma2(*reinterpret_cast<const Two*>(&a), *reinterpret_cast<const Two*>(&b), *reinterpret_cast<const Two*>(&c));
  return *reinterpret_cast<const uint32_t*>(&d);
}
template <typename T>
__device__ __forceinline__ uint32_t bits16(T x) {
  return *reinterpret_cast<const uint16_t*>(&x);
}

// x c + y s of 16-bit x and y, rounded once.  32 bits give it to one unit in their
// last place (what the rounding of y s lost is added), so if a unit up and a
// unit down round to the same 16 bits, that is the answer; in one of 20,000
// (fp16: of 2,700) they do not, and 64 bits, which hold both products, decide.  So a quantised cache's codes
// do not hang on how an angle's product was rounded.  (Where bfloat16's subnormals
// are cut off from those of 32 bits, below 2^-126, the last step may be off.)
template <typename T>
__device__ __noinline__ uint32_t turn_wide(float x, float c, float y, float s) {
  return bits16(Half16<T>::put((double)x * (double)c + (double)y * (double)s));
}
// Eight channels as pairs w, and their partners p; s has the sign of its channel
// changed.
template <typename T>
__device__ __forceinline__ void turn8(uint32_t (&w)[4], const uint32_t (&p)[4], const float2 (&c)[4], const float2 (&s)[4]) {
  using Two = typename Half16<T>::Two;
  uint32_t up[4], bad[4], any = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 x = Half16<T>::get2(w[k]), y = Half16<T>::get2(p[k]);
    const float2 q = mul2(y, s[k]), e = fma2(y, s[k], mul2(q, both(-1.f)));  // y s, and what its rounding lost
    const float2 z = add2(fma2(x, c[k], q), e);
    const float2 a = mul2(z, both(1.f + 0x1p-23f)), b = mul2(z, both(1.f - 0x1p-23f));
    up[k] = Half16<T>::pack(a.x, a.y);
    const uint32_t down = Half16<T>::pack(b.x, b.y);
    // (an infinity or NaN may be what is left of an infinite product)
    bad[k] = (up[k] ^ down) | (fma_bits<Two>(up[k], 0u, 0u) & 0x7FFF7FFFu);
    any |= bad[k];
  }
  if (any) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (bad[k]) {
        const float2 x = Half16<T>::get2(w[k]), y = Half16<T>::get2(p[k]);
        up[k] = turn_wide<T>(x.x, c[k].x, y.x, s[k].x) | turn_wide<T>(x.y, c[k].y, y.y, s[k].y) << 16;
      }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = up[k];
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
