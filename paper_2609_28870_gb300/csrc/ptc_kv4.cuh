// Pages of 4 bits: a row's layout, and its values.
//
// A row of up to 64 (128) channels is 48 (80) bytes: 8 (16) words of codes,
// then 2 (4) words of scale and base, one for 32 channels, then nothing up to a
// multiple of 16 bytes.  Word i holds channels 8 i .. 8 i + 7, the even ones in
// its low half and the odd ones in its high half, four bits each from the
// lowest: one shift and one mask of a word give two neighbours, each in its own
// half, as a pair of 16-bit numbers wants them.  Of a word (scale, base) the
// scale is the low half.
//
//   value = (16 + code) * scale + base, rounded to the cache's 16-bit type
//
// 16 + code is a 16-bit number whose exponent is 16's and whose upper mantissa
// bits are the code, so it is made by or-ing the shifted code into 16, and two
// values by one fused multiply-add; the base absorbs the 16.  A value is a
// 16-bit number by definition, so the matrix products that take it lose nothing.
#pragma once

#include "ptc_rope.cuh"

namespace ptc {

constexpr uint32_t kGroup4 = 32;  // channels of a scale and base
__host__ __device__ constexpr uint32_t padded4(uint32_t D) { return D <= 64 ? 64 : 128; }
__host__ __device__ constexpr uint32_t row4_bytes(uint32_t D) { return D <= 64 ? 48 : 80; }

// The pair `j` of a word's channels (2 j and 2 j + 1) as numbers 16 + code.
template <typename T>
__device__ __forceinline__ uint32_t pair4(uint32_t w, int j) {
  constexpr int at = Half16<T>::kBf16 ? 3 : 6;  // the code's place among the mantissa bits
  constexpr uint32_t mask = 0xFu << at | 0xFu << (at + 16), one = Half16<T>::kBf16 ? 0x41804180u : 0x4C004C00u;
  const int up = at - 4 * j;
  // (one instruction: left to itself the compiler takes two, each with a constant of its own)
  uint32_t y;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(y) : "r"(up >= 0 ? w << up : w >> -up), "r"(mask), "r"(one));
  return y;
}
template <typename T>
__device__ __forceinline__ uint32_t fma16x2(uint32_t a, uint32_t b, uint32_t c) {
  return fma_bits<typename Half16<T>::Two>(a, b, c);
}
__device__ __forceinline__ uint32_t both_low(uint32_t x) { return __byte_perm(x, x, 0x1010); }
__device__ __forceinline__ uint32_t both_high(uint32_t x) { return __byte_perm(x, x, 0x3232); }

// key / B as (key * mul >> 32) >> shift, exact for keys below 2^31 and B > 1: mul's
// error, below B, times key is below 2^32 << shift, as B <= 2 << shift.
inline void page_division(uint32_t B, uint32_t* mul, uint32_t* shift) {
  *shift = 0;
  while (B > 2u << *shift) ++*shift;
  *mul = B > 1 ? (uint32_t)(((uint64_t(1) << (32 + *shift)) + B - 1) / B) : 0;
}

// The host-side checks of a ptc_paged_kv whose pages are 4-bit rows, and its
// device view; strides in bytes.
inline ptc_status kv4_view(const ptc_paged_kv* kv, KvView* o) {
  if (!kv) return PTC_ERR_INVALID_ARG;
  const uint32_t ext[3] = {kv->n_pages, kv->n_kv_heads, kv->block_size};
  for (int i = 0; i < 3; ++i)
    if ((ext[i] > 1 && kv->k_stride[i] % 16) || (ext[i] > 1 && kv->v_stride[i] % 16)) return PTC_ERR_INVALID_ARG;
  const ptc_status st = kv_view(kv, o);
  if (st != PTC_OK) return st;
  // (the stride of a dimension of size 1 is not used, but tensor maps want a multiple of 16)
  int64_t* s[6] = {&o->ks_page, &o->ks_head, &o->ks_slot, &o->vs_page, &o->vs_head, &o->vs_slot};
  for (int i = 0; i < 6; ++i)
    if (ext[i % 3] <= 1) *s[i] = 16;
  return PTC_OK;
}

}  // namespace ptc
