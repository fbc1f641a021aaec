// Attention by tiles of 256 query rows and 128 keys on the tensor cores, over
// pages of 16 bits (ptc_attn.cu) or of 4 (ptc_attn4.cu).
#pragma once

#include "ptc_attn.cuh"
#include "ptc_kv4.cuh"

namespace ptc {
namespace {

// The query tiles that a CTA has a part in, in order, with the part.
struct Walk {
  uint64_t left, u, tok0, page0;     // units left, the part's first unit
  uint32_t r, h, qt, kv0, kv1, nkv;  // key tiles [kv0, kv1) of nkv
  uint32_t extra;                    // units before the first key tile
  uint32_t m, n;
  bool first;                        // the CTA's first part
  __device__ __forceinline__ void request(const AttnArgs& a) {
    tok0 = a.tok_off[r];
    m = (uint32_t)(a.tok_off[r + 1] - tok0);
    n = a.kv.kv_len[r];
    page0 = a.kv.page_off[r];
  }
  __device__ __forceinline__ uint32_t cost(const AttnArgs& a) const { return tile_extra(m, 2 * a.tq, a.tq32, qt); }
  __device__ __forceinline__ void part(const AttnArgs& a) {
    nkv = key_tiles(m, n, 2 * a.tq, qt);
    extra = kv0 ? 0 : cost(a);
    kv1 = nkv - kv0 + extra > left ? kv0 + (uint32_t)left - extra : nkv;
  }
  // The next query tile.
  __device__ __forceinline__ bool step(const AttnArgs& a) {
    kv0 = 0;
    if (++qt * 2 * a.tq >= m) {
      qt = 0;
      if (++h == a.kv.H) {
        h = 0;
        do {
          if (++r == a.kv.n_req) return false;
          request(a);
        } while (m == 0);
      }
    }
    return true;
  }
  // False if the CTA has nothing to do.
  __device__ __forceinline__ bool begin(const AttnArgs& a) {
    const CtaStart* start = a.plan->start + blockIdx.x;
    const CtaStart s = start[0];
    left = start[1].u - s.u;
    if (left == 0) return false;
    u = s.u;
    first = true;
    r = s.r;
    h = s.h;
    qt = s.major;
    kv0 = s.minor;
    tok0 = s.tok0;
    m = s.m;
    n = s.n;
    page0 = s.page0;
    if (kv0 && kv0 == key_tiles(m, n, 2 * a.tq, qt) && !step(a)) return false;
    part(a);
    return true;
  }
  __device__ __forceinline__ bool next(const AttnArgs& a) {
    const uint32_t had = kv1 - kv0 + extra;
    left -= had;
    u += had;
    first = false;
    if (left == 0 || !step(a)) return false;
    part(a);
    return true;
  }
  // The tile's first token.
  __device__ __forceinline__ uint32_t token0(const AttnArgs& a) const { return qt * 2 * a.tq; }
  // The units of the whole tile.
  __device__ __forceinline__ uint64_t from(const AttnArgs& a) const { return kv0 ? u - kv0 - cost(a) : u; }
  __device__ __forceinline__ uint64_t to(const AttnArgs& a) const { return from(a) + cost(a) + nkv; }
  // How the two halves of the softmax share the tile.
  __device__ __forceinline__ int mode(const AttnArgs& a) const {
    const uint32_t tokens = m - token0(a);
    return tokens > a.tq ? 0 : tokens > a.tq32 ? 1 : 2;
  }
};

// Two 32-bit floats rounded to the cache's type, the first in the low half.
// Attention weights of bf16 caches are rounded as they are.  Those of fp16
// caches are scaled by 2^7 first: a weight far below the running maximum would
// otherwise fall among fp16's subnormals (below 2^-14) and a long row of small
// weights would be lost; with kMove's 2^8 the largest is 2^15.
template <typename T>
struct Weights;
template <>
struct Weights<__nv_bfloat16> {
  static constexpr bool kBf16 = true;
  static constexpr float kShift = 0.f, kScale = 1.f;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
};
template <>
struct Weights<__half> {
  static constexpr bool kBf16 = false;
  static constexpr float kShift = 7.f, kScale = 128.f;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 x = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
};

// ------------------------------------------------------------------ the tile kernel
// One CTA an SM walks its units.  Warps 0-3 and 4-7 are the two halves of the
// softmax, warp 8 issues the products, warp 9 loads keys and warp 11 values into
// a ring of tiles, warp 10 loads the queries of the next tile.  (Pages of 16 are 16
// copies a tile: one warp for both took 179 us for 64 single tokens, two 158;
// 1.31 and 1.23 ms for 4,096 tokens at 32K.)  For key tile j:
//   scores   S = Q K_j^T     128 x 128 sums in tensor memory
//   softmax  one thread a row: running maximum and sum in 32 bits; weights
//            exp2(s - max), rounded to 16 bits, over the scores' columns
//   values   O += P V_j      P from tensor memory, O stays there
// While one half is in its softmax, the tensor cores work for the other:
//   kRowsApart    more than 128 rows: each half has its own rows and takes
//                 every key tile
//   kTilesApart   up to 128 rows: both halves have the same rows and take key
//                 tiles in turn; two partial rows are put together at the end
//   kColumnsApart up to 32 rows (single tokens): the rows stand four times in
//                 the matrix, and each of the 4 warps takes 32 keys of a tile,
//                 with zero weights for the others'.  A softmax over 32 keys is
//                 a quarter of the latency that a tile waits for (64 single
//                 tokens: 307 us with whole rows, 204 so); the products are the
//                 same instructions either way.
// The maximum that weights are taken with need not be the row's: weights up to
// 2^8 are as exact as those up to 1.  So it is only looked for, and O only
// rescaled, when 64 weights add up to more than 2^8, which after the first tile
// hardly happens (2.02 -> 1.38 ms for 4,096 tokens at 32K, with the products'
// descriptors made outside the issuing lane).
//
// Bounds.  Single tokens: HBM; 12 contexts of 32K to 131K, 1.81 GB, take 275 us,
// 6.6 TB/s.  Chunks: the tensor cores; a unit of 256 rows and 128 keys is 2,048
// cycles of products at D = 128 and takes 2,700 (4,096 tokens at 32K: 1.22 ms in
// a few calls, 1.69 PFLOP/s, the tensor pipe 75% active at 1.84 GHz; 1.37 ms,
// 1.50 PFLOP/s, in many, where the power cap takes the clock down).  A half's own
// chain (softmax 1,260, its two products 1,024, four hand-overs) is 2,600, and
// what the products and copies move through shared memory, 256 KB, 2,048 cycles
// at 128 bytes a cycle.  At D <= 64 a unit takes 2,600 cycles for 1,024 of
// products and 1,024 of exponentials: the softmax's chain alone (2,048 tokens at
// 20K, 32 heads of 64: 387 us for 182 of products).  Short query tiles: their
// way out and the joins (40 prompts of 100 to 300 tokens 75 us for 23).
enum { kRowsApart = 0, kTilesApart = 1, kColumnsApart = 2 };
constexpr int kTileThreads = 384;
constexpr int kSlabBytes = 128 * 128;  // 128 rows of 64 columns
// 4 KB a softmax warp: rows on their way out; the sums of 8 warps, 32 rows and 32 columns.
constexpr int kStage = 8 * 4096;
// Registers a thread: 2 * 128 * 200 + 128 * 104 = 384 * 168, what the block has at launch.
// With four warps more: 256 * 184 + 256 * 72 = 512 * 128 (4,096 tokens at 32K: 1.47 ms;
// with 200, 56 and 56 2.0 ms, the copies' state in local memory).
constexpr int kSoftmaxRegs = 200, kOtherRegs = 104, kSoftmaxRegs4 = 184, kOtherRegs4 = 72, kQuantRegs4 = 72;

struct TileShared {
  uint64_t full[8], empty[8], q_full[2], q_empty[2], s_full[2], p_full[2][2], pv_done[2][2], drain;
  float2 ml[256];
  uint32_t tmem, last, count, c0;
  uint32_t issued[2], loads[2];  // tensor copies of keys and of values, loads of either half's queries
  uint16_t slots[kMaxCtas];  // a split tile's parts, in the order of the keys
};

// Kinds of the kernel.
//   kFew   every request of the call has so few rows that its tiles are all
//          kColumnsApart.  There is no second half of queries then, and the
//          ring has its place: 5 tiles of 32 KB keep more of the cache in
//          flight than 4.
//   kFour  the cache is of 4 bits: warps 12-15 take the place of 9 and 11, see
//          quant_role.  What is in flight waits in 4 bits, so the ring of
//          tiles may be short.
enum { kAny = 0, kFew = 1, kFour = 2 };
template <int NSLAB, int KIND>
struct TileShape {
  static constexpr int kTile = NSLAB * kSlabBytes;
  static constexpr uint32_t kRing = KIND == kFour ? (NSLAB == 1 ? 6 : 3) : NSLAB == 1 ? 8 : KIND == kFew ? 5 : 4;
  static constexpr int kQueries = KIND == kFew ? 1 : 2;
  // tiles of 4 bits
  static constexpr uint32_t kRow4 = NSLAB == 1 ? 48 : 80, kRing4 = NSLAB == 1 ? 4 : 3;
  static constexpr int kTiles4 = KIND == kFour ? kRing4 * 128 * kRow4 : 0;
  // A role's warps, and registers a thread: the softmax's and the others'.
  static constexpr int kThreads = KIND == kFour ? 512 : kTileThreads;
  static constexpr int kSoftmax = KIND == kFour ? kSoftmaxRegs4 : kSoftmaxRegs, kOther = KIND == kFour ? kOtherRegs4 : kOtherRegs;
  // queries, ring, tiles of 4 bits, stage, the rest
  static constexpr int kRest = kQueries * kTile + kRing * kTile + kTiles4 + kStage;
  static constexpr int kSmem = kRest + sizeof(TileShared) + (KIND == kFour ? 4 * sizeof(Walk) : 0);
  static_assert(kSmem <= 227 * 1024, "shared memory of a block");
};

// Tensor memory columns: scores of both halves, then their sums.  The weights
// of keys 0-63 and of keys 64-127 lie in the first 32 columns of their own scores.
__device__ __forceinline__ uint32_t s_col(uint32_t half) { return half * 128; }
__device__ __forceinline__ uint32_t o_col(uint32_t half) { return 256 + half * 128; }
__device__ __forceinline__ uint32_t p_col(uint32_t half, uint32_t key) { return half * 128 + (key & 64) + (key & 63) / 2; }

// Both halves of the softmax.
__device__ __forceinline__ void softmax_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// 128 bytes a lane to the lanes' places in global memory, `pieces` of 16 bytes
// of each, by way of the warp's stage: a store then covers 128 bytes of 4 rows
// and not 16 of 32 (which made this a third of the time of a short tile).
__device__ __forceinline__ void emit(char* stage, const uint4 (&x)[8], char* to, uint32_t rows, uint32_t pieces) {
  const uint32_t lane = threadIdx.x & 31;
#pragma unroll
  for (uint32_t k = 0; k < 8; ++k) *reinterpret_cast<uint4*>(stage + lane * 128 + (k ^ (lane & 7)) * 16) = x[k];
  __syncwarp();
#pragma unroll
  for (uint32_t i = 0; i < 8; ++i) {
    const uint32_t row = i * 4 + lane / 8, k = lane & 7;
    const uint4 y = *reinterpret_cast<const uint4*>(stage + row * 128 + (k ^ (row & 7)) * 16);
    char* p = reinterpret_cast<char*>(__shfl_sync(kFull, reinterpret_cast<uint64_t>(to), row));
    if ((rows >> row & 1) && k < pieces) *reinterpret_cast<uint4*>(p + 16 * k) = y;
  }
  __syncwarp();
}

// The running maximum and sum of a row.
struct RowState {
  float top, l;
  __device__ __forceinline__ void clear() {
    top = -INFINITY;
    l = 0.f;
  }
  // The maximum as a power of two, as the weights were scaled by it.
  template <typename W>
  __device__ __forceinline__ float top2(float sl2) const {
    return l != 0.f ? top * sl2 - W::kShift : -INFINITY;  // a NaN sum is not an empty one
  }
};

// Moves the maximum of a row up to mx; O, once the product before is done,
// and what was summed so far shrink with it.
template <int NSLAB>
__device__ __forceinline__ void raise_top(RowState& st, float mx, float sl2, uint32_t o_at, bool first,
                                          uint32_t bar_o, uint32_t parity, long long limit, bool& alive) {
  if (!__any_sync(kFull, mx > st.top)) return;
  const float nt = fmaxf(st.top, mx);
  const float f = st.top == -INFINITY ? 0.f : exp2_approx((st.top - nt) * sl2);
  st.l *= f;
  st.top = nt;
  if (first) return;
  if (alive) alive = mbar_wait(bar_o, parity, limit);
  tc_fence_after();
#pragma unroll 1
  for (int c = 0; c < NSLAB * 2; ++c) {
    uint32_t x[32];
    tmem_ld32(x, o_at + 32 * c);
    tmem_wait_ld(x);
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * f);
    tmem_st32(o_at + 32 * c, x);
  }
}

__device__ __forceinline__ float max32(const uint32_t (&x)[32]) {
  float m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = __uint_as_float(x[i]);
#pragma unroll
    for (int k = i + 4; k + 4 < 32; k += 8)
      m[i] = fmaxf(m[i], fmaxf(__uint_as_float(x[k]), __uint_as_float(x[k + 4])));
    m[i] = fmaxf(m[i], __uint_as_float(x[i + 28]));
  }
  return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
}

// A sum in eight strands: with four, the additions' latency is what a warp
// waits for (254 cycles for 32 weights against 176, alone on its scheduler).
struct Sums {
  float2 s[4];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = make_float2(0.f, 0.f);
  }
  __device__ __forceinline__ void add(int i, float2 x) { s[i & 3] = add2(s[i & 3], x); }
  __device__ __forceinline__ float total() const {
    const float2 t = add2(add2(s[0], s[1]), add2(s[2], s[3]));
    return t.x + t.y;
  }
};

// 32 scores to weights: their sum, and the weights in 16 columns.
template <typename T>
__device__ __forceinline__ void weigh(const uint32_t (&x)[32], float sl2, float sub, Sums& sum, uint32_t (&y)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float2 e = fma2(make_float2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), make_float2(sl2, sl2),
                          make_float2(-sub, -sub));
    const float2 p = make_float2(exp2_approx(e.x), exp2_approx(e.y));
    sum.add(i, p);
    y[i] = Weights<T>::pack(p.x, p.y);
  }
}

// The maximum moves when a row's sum of 64 (or 32) weights passes this: as many
// of at most 1 stay below it, and no weight is larger than their sum.  (For fp16
// the weights, and with them this, are 2^7 times as large.)
constexpr float kMove = 256.f;

// Who has a part of the tile, and where; by one warp.
__device__ __noinline__ void list_sharers(const AttnArgs& a, TileShared& sh, uint64_t from, uint64_t to) {
  const uint32_t lane = threadIdx.x & 31;
  const AttnPlan* plan = a.plan;
  const Sharers s = sharers(plan, a.ctas, from, to);
  uint32_t n = 0;
  for (uint32_t x0 = s.c0; x0 <= s.c1; x0 += 32) {
    const uint32_t x = x0 + lane;
    const uint64_t u = x <= s.c1 ? plan->start[x].u : 0, v = x <= s.c1 ? plan->start[x + 1].u : 0;
    const uint32_t has = __ballot_sync(kFull, v > u);
    // a CTA's first part, or (of the tile's first CTA, where it began with another tile) its last
    if (v > u) sh.slots[n + __popc(has & ((1u << lane) - 1))] =
          (uint16_t)(2 * x + (u < from ? 1 : 0));
    n += __popc(has);
  }
  if (lane == 0) {
    sh.c0 = s.c0;
    sh.count = s.count;
  }
  __syncwarp();
}

// The parts of a split tile put together, by all of the softmax: a warp takes
// ROWS rows at a time.  Lane p looks at part p's maximum and sum of a row; then
// the lanes have 4 columns each, and the parts are added up in the order of the
// keys.
template <typename T, int ROWS>
__device__ __noinline__ void join_parts(const AttnArgs& a, const TileShared& sh, uint64_t tok0, uint32_t m, uint32_t t0,
                                        uint32_t h) {
  const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = a.kv.D, count = sh.count;
  const bool in = 4 * lane < D;
  for (uint32_t i0 = warp * ROWS; i0 < (ROWS == 1 ? 32 : kRows); i0 += 8 * ROWS) {
    bool ok[ROWS];
    uint64_t at[ROWS];
    float top[ROWS], l[ROWS];
    float2 ml[ROWS];
    float4 o[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      // row i of the tile: its half, token and head
      const uint32_t i = (i0 + k) & 127, t = t0 + ((i0 + k) >> 7) * a.tq + i / a.G;
      ok[k] = i < a.tq * a.G && t < m;
      at[k] = (tok0 + t) * a.n_q_heads + h * a.G + i % a.G;
      top[k] = -INFINITY;
      l[k] = 0.f;
      o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    if (!ok[0]) continue;  // rows of a half are none from some row on
    auto look = [&](uint32_t p0) {
#pragma unroll
      for (int k = 0; k < ROWS; ++k)
        ml[k] = p0 + lane < count ? __ldcg(a.part_ml + sh.slots[p0 + lane] * kRows + i0 + k) : make_float2(-INFINITY, 0.f);
    };
    for (uint32_t p0 = 0; p0 < count; p0 += 32) {
      look(p0);
#pragma unroll
      for (int k = 0; k < ROWS; ++k) {
        float mx = ml[k].x;
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, x));
        const float nt = fmaxf(top[k], mx), base = nt == -INFINITY ? 0.f : nt;
        float sum = ml[k].x == -INFINITY ? 0.f : ml[k].y * exp2_approx(ml[k].x - base);
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(kFull, sum, x);
        l[k] = l[k] * exp2_approx(top[k] - base) + sum;
        top[k] = nt;
      }
    }
    for (uint32_t p0 = 0; p0 < count; p0 += 32) {
      if (count > 32) look(p0);
      float f[ROWS];
#pragma unroll
      for (int k = 0; k < ROWS; ++k) f[k] = ml[k].x == -INFINITY ? 0.f : exp2_approx(ml[k].x - top[k]) / l[k];
      const uint32_t n = count - p0 < 32 ? count - p0 : 32;
#pragma unroll (8 / ROWS)
      for (uint32_t p = 0; p < n; ++p) {
        const float* row = a.part + ((uint64_t)sh.slots[p0 + p] * kRows + i0) * D + 4 * lane;
        float4 x[ROWS];
#pragma unroll
        for (int k = 0; k < ROWS; ++k)  // (a part's place has all kRows rows; those that are none are not used)
          x[k] = in ? __ldcg(reinterpret_cast<const float4*>(row + k * D)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
          const float fp = __shfl_sync(kFull, f[k], p);
          if (fp == 0.f) continue;  // the row saw no key of the part
          o[k].x = fmaf(x[k].x, fp, o[k].x);
          o[k].y = fmaf(x[k].y, fp, o[k].y);
          o[k].z = fmaf(x[k].z, fp, o[k].z);
          o[k].w = fmaf(x[k].w, fp, o[k].w);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      if (ok[k] && in)
        *reinterpret_cast<uint2*>(a.out + 2 * (at[k] * D + 4 * lane)) =
            make_uint2(Weights<T>::pack(o[k].x, o[k].y), Weights<T>::pack(o[k].z, o[k].w));
      if (ok[k] && lane == 0) a.lse[at[k]] = top[k] == -INFINITY ? -INFINITY : (top[k] + log2_approx(l[k])) * kLn2;
    }
  }
}

template <typename T, int NSLAB, int KIND>
__device__ __forceinline__ bool softmax_role(const AttnArgs& a, TileShared& sh, char* stages, uint32_t half) {
  using W = Weights<T>;
  const uint32_t tid = threadIdx.x & 127, lane = tid & 31, warp = tid >> 5;
  const uint32_t tmem = sh.tmem + ((tid & ~31u) << 16);
  const uint32_t s_at = tmem + s_col(half), o_at = tmem + o_col(half);
  const uint32_t bar_s = smem_u32(&sh.s_full[half]);
  const uint32_t bar_p[2] = {smem_u32(&sh.p_full[half][0]), smem_u32(&sh.p_full[half][1])};
  const uint32_t bar_o[2] = {smem_u32(&sh.pv_done[half][0]), smem_u32(&sh.pv_done[half][1])};
  const float sl2 = a.scale * kLog2e;
  const uint32_t D = a.kv.D, G = a.G;
  char* stage = stages + (half * 4 + warp) * 4096;
  bool alive = true;  // a warp that has given up waiting runs on without, for the others at the barriers
  uint32_t done = 0, parted = 0;  // key tiles of this half so far, and those in two parts
  Walk w;
  for (bool more = w.begin(a); more; more = w.next(a)) {
    const int mode = KIND == kFew ? kColumnsApart : w.mode(a);
    // the thread's row: a token of the request and a head of the group
    const uint32_t i = mode == kColumnsApart ? lane : tid;
    const uint32_t t = w.token0(a) + (mode == kRowsApart ? half * a.tq : 0) + i / G, g = i % G;
    const bool valid = i < a.tq * G && t < w.m;
    const uint32_t rows = __ballot_sync(kFull, valid);
    const uint32_t step = mode == kRowsApart ? 1 : 2, j0 = w.kv0 + (mode == kRowsApart ? 0 : half);
    // keys of the tile at hand and later ones that the row sees; what a row
    // computes that is none is not used and moves nothing
    int64_t see_all = valid ? (int64_t)w.n - w.m + t + 1 - (int64_t)j0 * kKeys : INT64_MAX / 2;
    RowState st;
    st.clear();
    const bool whole = w.kv0 == 0 && w.kv1 == w.nkv;
    if (!whole && threadIdx.x < 32) list_sharers(a, sh, w.from(a), w.to(a));
    if (mode != kColumnsApart) {
      for (uint32_t j = j0; j < w.kv1; j += step, ++done, ++parted, see_all -= step * kKeys) {
        if (alive) alive = mbar_wait(bar_s, done & 1, a.limit);
        tc_fence_after();
        const int see = see_all >= (int64_t)kKeys ? (int)kKeys : see_all > 0 ? (int)see_all : 0;
        const bool masked = __any_sync(kFull, see < (int)kKeys);
        uint32_t x[4][32];
        if (rows) {
          tmem_ld32(x[0], s_at);
          tmem_ld32(x[1], s_at + 32);
        }
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          if (rows) {
            const uint32_t x_at = s_at + 64 * part;
            uint32_t y[16];
            Sums sum;
            sum.clear();
            float sub = (st.top == -INFINITY ? 0.f : st.top * sl2) - W::kShift;
            const bool first = j == j0 && part == 0;
            tmem_wait_ld(x[2 * part]);
            tmem_wait_ld(x[2 * part + 1]);
            if (part == 0) {  // the second part's scores come in behind the first's weights
              tmem_ld32(x[2], s_at + 64);
              tmem_ld32(x[3], s_at + 96);
            }
            if (masked) {
#pragma unroll
              for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int k = 0; k < 32; ++k)
                  if (64 * part + 32 * c + k >= see) x[2 * part + c][k] = 0xFF800000u;
            }
            bool move = first;
            if (!first) {
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                weigh<T>(x[2 * part + c], sl2, sub, sum, y);
                tmem_st16(x_at + 16 * c, y);
              }
              const float total = sum.total();
              move = __any_sync(kFull, valid && !(total <= kMove * W::kScale));
              if (!move) st.l += total;
            }
            if (move) {
              const float mx = valid ? fmaxf(max32(x[2 * part]), max32(x[2 * part + 1])) : -INFINITY;
              raise_top<NSLAB>(st, mx, sl2, o_at, first, bar_o[1 - part], (part ? parted : done - 1) & 1, a.limit,
                               alive);
              sub = (st.top == -INFINITY ? 0.f : st.top * sl2) - W::kShift;
              sum.clear();
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                weigh<T>(x[2 * part + c], sl2, sub, sum, y);
                tmem_st16(x_at + 16 * c, y);
              }
              st.l += sum.total();
            }
            tmem_wait_st();
          }
          tc_fence_before();
          mbar_arrive_warp(bar_p[part]);
        }
      }
    } else {
      see_all -= 32 * warp;
      for (uint32_t j = j0; j < w.kv1; j += step, ++done, see_all -= step * kKeys) {
        if (alive) alive = mbar_wait(bar_s, done & 1, a.limit);
        tc_fence_after();
        uint32_t x[32], y[16], zero[16];
        tmem_ld32(x, s_at + 32 * warp);
        tmem_wait_ld(x);
        const int see = see_all >= 32 ? 32 : see_all > 0 ? (int)see_all : 0;
        if (a.scores && valid) {
          float* to = a.scores + ((uint64_t)w.h * a.few + lane) * a.mass_stride + w.page0 * a.kv.B + (uint64_t)j * kKeys + 32 * warp;
          if (see == 32 && (a.mass_stride & 3) == 0 && (w.page0 * a.kv.B & 3) == 0) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
              *reinterpret_cast<uint4*>(to + 4 * k) = make_uint4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
          } else {
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if (k < see) to[k] = __uint_as_float(x[k]);
          }
        }
        __syncwarp();
        if (__any_sync(kFull, see < 32)) {
#pragma unroll
          for (int k = 0; k < 32; ++k)
            if (k >= see) x[k] = 0xFF800000u;
        }
        float sub = (st.top == -INFINITY ? 0.f : st.top * sl2) - W::kShift;
        Sums sum;
        sum.clear();
        weigh<T>(x, sl2, sub, sum, y);
        float total = sum.total();
        if (__any_sync(kFull, j == j0 || (valid && !(total <= kMove * W::kScale)))) {
          raise_top<NSLAB>(st, valid ? max32(x) : -INFINITY, sl2, o_at, j == j0, bar_o[1], (done - 1) & 1, a.limit,
                             alive);
          sub = (st.top == -INFINITY ? 0.f : st.top * sl2) - W::kShift;
          sum.clear();
          weigh<T>(x, sl2, sub, sum, y);
          total = sum.total();
        }
        st.l += total;
#pragma unroll
        for (int k = 0; k < 16; ++k) zero[k] = 0;
#pragma unroll
        for (uint32_t c = 0; c < 4; ++c) {
          if (c == warp) tmem_st16(tmem + p_col(half, 32 * c), y);
          else tmem_st16(tmem + p_col(half, 32 * c), zero);
        }
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive_warp(bar_p[1]);
      }
    }
    // the sums of the rows
    const bool some = j0 < w.kv1;  // this half had a key tile
    if (some && alive) alive = mbar_wait(bar_o[1], (done - 1) & 1, a.limit);
    tc_fence_after();
    const uint64_t prow0 = (uint64_t)(2 * blockIdx.x + (w.first ? 0 : 1)) * kRows;
    const uint64_t orow0 = w.tok0 * a.n_q_heads + w.h * G;  // row (t, g) is orow0 + t * n_q_heads + g
    if (mode != kColumnsApart) {
      float top2 = st.top2<W>(sl2), l = st.l, f0 = 1.f, f1 = 0.f;
      if (mode == kTilesApart) {
        if (half == 1) sh.ml[tid] = make_float2(top2, l);
        softmax_sync();
        if (half == 0) {
          const float2 other = sh.ml[tid];
          const float m2 = fmaxf(top2, other.x);
          f0 = top2 == -INFINITY ? 0.f : exp2_approx(top2 - m2);
          f1 = other.x == -INFINITY ? 0.f : exp2_approx(other.x - m2);
          top2 = m2;
          l = l * f0 + (other.x == -INFINITY ? 0.f : other.y * f1);
        }
      }
      if (rows && (mode == kRowsApart || half == 0)) {
        const bool none = top2 == -INFINITY;
        const float inv = whole ? 1.f / l : 1.f;
        f0 *= inv;
        f1 *= inv;
        const uint64_t at = orow0 + (uint64_t)t * a.n_q_heads + g, prow = prow0 + (mode == kRowsApart ? half * 128 : 0) + i;
        const bool two = mode == kTilesApart && w.kv1 - w.kv0 > 1;
        auto sums_of = [&](uint32_t col, uint32_t(&x)[32]) {
          tmem_ld32(x, o_at + col);
          tmem_wait_ld(x);
#pragma unroll
          for (int k = 0; k < 32; ++k) x[k] = none || f0 == 0.f ? 0u : __float_as_uint(__uint_as_float(x[k]) * f0);
          if (two) {
            uint32_t z[32];
            tmem_ld32(z, tmem + o_col(1) + col);
            tmem_wait_ld(z);
#pragma unroll
            for (int k = 0; k < 32; ++k)
              if (!none && f1 != 0.f) x[k] = __float_as_uint(fmaf(__uint_as_float(z[k]), f1, __uint_as_float(x[k])));
          }
        };
        if (whole) {
#pragma unroll 1
          for (uint32_t col = 0; col < NSLAB * 64; col += 64) {
            uint4 y[8];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              uint32_t x[32];
              sums_of(col + 32 * c, x);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                auto two16 = [&](int e) { return W::pack(__uint_as_float(x[8 * k + e]), __uint_as_float(x[8 * k + e + 1])); };
                y[4 * c + k] = make_uint4(two16(0), two16(2), two16(4), two16(6));
              }
            }
            emit(stage, y, a.out + 2 * (at * D + col), rows, (D - col) / 8);
          }
        } else {
#pragma unroll 1
          for (uint32_t col = 0; col < D; col += 32) {
            uint32_t x[32];
            sums_of(col, x);
            uint4 y[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) y[k] = make_uint4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
            emit(stage, y, reinterpret_cast<char*>(a.part + prow * D + col), rows, (D - col) / 4);
          }
        }
        if (valid) {
          if (whole) a.lse[at] = none ? -INFINITY : (top2 + log2_approx(l)) * kLn2;
          else a.part_ml[prow] = make_float2(top2, l);
        }
      }
      tc_fence_before();
      if (mode == kTilesApart) softmax_sync();  // half 1's sums have been read
    } else {
      // the eight partial rows of a row
      const uint32_t count = (w.m - w.token0(a)) * G, w8 = half * 4 + warp;
      sh.ml[w8 * 32 + lane] = make_float2(st.top2<W>(sl2), st.l);
      softmax_sync();
      float top2 = -INFINITY, l = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) top2 = fmaxf(top2, sh.ml[k * 32 + lane].x);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float2 ml = sh.ml[k * 32 + lane];
        if (ml.x != -INFINITY) l = fmaf(ml.y, exp2_approx(ml.x - top2), l);
      }
      const bool none = top2 == -INFINITY;
      const float mine = st.top2<W>(sl2);
      float f = mine == -INFINITY ? 0.f : exp2_approx(mine - top2);
      if (whole && !none) f *= 1.f / l;
      if (w8 == 0 && valid) {
        if (whole) a.lse[orow0 + (uint64_t)t * a.n_q_heads + g] = none ? -INFINITY : (top2 + log2_approx(l)) * kLn2;
        else a.part_ml[prow0 + lane] = make_float2(top2, l);
      }
      // columns at a time that fit the stage: [8 warps][rows][cols], or
      // [8][rows][32] where there are many rows
      const uint32_t cols = count <= 8 ? NSLAB * 64 : 32;
      float* buf = reinterpret_cast<float*>(stages);
      for (uint32_t c0 = 0; c0 < NSLAB * 64; c0 += cols) {
#pragma unroll 1
        for (uint32_t c = 0; c < cols; c += 32) {
          uint32_t x[32];
          tmem_ld32(x, o_at + c0 + c);
          tmem_wait_ld(x);
          if (lane < count) {
            float4* to = reinterpret_cast<float4*>(buf + ((uint64_t)w8 * count + lane) * cols + c);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              // rotated by the row: the lanes' rows are whole multiples of the banks apart
              const uint32_t at = (k + lane) & 7;
              float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
              if (f != 0.f)
                y = make_float4(__uint_as_float(x[4 * k]) * f, __uint_as_float(x[4 * k + 1]) * f,
                                __uint_as_float(x[4 * k + 2]) * f, __uint_as_float(x[4 * k + 3]) * f);
              to[at] = y;
            }
          }
          __syncwarp();
        }
        tc_fence_before();
        softmax_sync();
        for (uint32_t e = threadIdx.x; e < count * (cols / 4); e += 256) {
          const uint32_t row = e / (cols / 4), c4 = e % (cols / 4);
          const uint32_t at = (c4 & ~7u) | ((c4 + row) & 7);
          float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float4 x = *reinterpret_cast<const float4*>(buf + ((uint64_t)k * count + row) * cols + 4 * at);
            y.x += x.x;
            y.y += x.y;
            y.z += x.z;
            y.w += x.w;
          }
          const uint32_t col = c0 + 4 * c4;
          if (col < D) {
            if (whole) {
              const uint64_t to = orow0 + (uint64_t)(w.token0(a) + row / G) * a.n_q_heads + row % G;
              *reinterpret_cast<uint2*>(a.out + 2 * (to * D + col)) = make_uint2(W::pack(y.x, y.y), W::pack(y.z, y.w));
            } else {
              *reinterpret_cast<float4*>(a.part + (prow0 + row) * D + col) = y;
            }
          }
        }
        softmax_sync();
      }
    }
    if (!whole) {
      // the last of the tile's CTAs to come here finds all parts in place
      __threadfence();
      softmax_sync();
      if (threadIdx.x == 0) {
        sh.last = atomicAdd(&a.plan->arrived[sh.c0], 1u) + 1 == sh.count;
        __threadfence();
      }
      softmax_sync();
      if (sh.last) {
        if (mode == kColumnsApart) join_parts<T, 1>(a, sh, w.tok0, w.m, w.token0(a), w.h);
        else join_parts<T, 4>(a, sh, w.tok0, w.m, w.token0(a), w.h);
      }
      softmax_sync();
    }
  }
  return alive;
}

template <typename T, int NSLAB, int KIND>
__device__ __forceinline__ bool product_role(const AttnArgs& a, TileShared& sh, uint32_t q_smem, uint32_t ring) {
  using Sh = TileShape<NSLAB, KIND>;
  constexpr uint32_t kQk = mma_desc(Weights<T>::kBf16, 128, kKeys, false);
  constexpr uint32_t kPv = mma_desc(Weights<T>::kBf16, 128, NSLAB * 64, true);
  const uint32_t lane = threadIdx.x & 31, tmem = sh.tmem, steps = (a.kv.D + 15) / 16;
  uint32_t item = 0;           // ring tiles before this query tile
  uint32_t used[2] = {0, 0};   // query tiles of each region
  uint32_t weights[2][2] = {};  // of each half: weights by part
  auto full = [&](uint32_t i) { return mbar_wait(smem_u32(&sh.full[i % Sh::kRing]), (i / Sh::kRing) & 1, a.limit); };
  auto tile_at = [&](uint32_t i) { return ring + (i % Sh::kRing) * Sh::kTile; };
  auto commit = [&](uint64_t& bar) {
    if (elect_lane()) mma_commit(smem_u32(&bar));
  };
  auto release = [&](uint32_t at) { mma_commit(smem_u32(&sh.empty[at])); };
  auto free_tile = [&](uint32_t i) {
    if (elect_lane()) release(i % Sh::kRing);
  };
  auto scores = [&](uint32_t half, uint32_t region, uint32_t k_item) {
    const uint64_t da = tile_desc(q_smem + region * Sh::kTile, 16), db = tile_desc(tile_at(k_item), 16);
    if (elect_lane()) {
      mma_ss<false>(tmem + s_col(half), da, db, kQk);
#pragma unroll
      for (uint32_t k = 1; k < NSLAB * 4; ++k) {
        const uint32_t off = (k / 4) * kSlabBytes + (k % 4) * 32;
        if (k < steps) mma_ss<true>(tmem + s_col(half), desc_at(da, off), desc_at(db, off), kQk);
      }
      mma_commit(smem_u32(&sh.s_full[half]));
    }
    __syncwarp();
  };
  // The weights of keys 0-63 and of 64-127 come one after the other (`apart`),
  // each as soon as it is there, or together.  Either way the second barrier
  // tells that the tile's product is done.
  auto values = [&](uint32_t half, uint32_t v_item, bool add, bool apart) {
    const uint64_t db = tile_desc(tile_at(v_item), kSlabBytes);
#pragma unroll
    for (uint32_t part = 0; part < 2; ++part) {
      if ((part || apart) && !mbar_wait(smem_u32(&sh.p_full[half][part]), weights[half][part]++ & 1, a.limit)) return false;
      if (!part && !apart) continue;
      tc_fence_after();
      if (elect_lane()) {
        if (part && !apart)
#pragma unroll
          for (uint32_t k = 0; k < 4; ++k)
            mma_ts(tmem + o_col(half), tmem + p_col(half, 16 * k), desc_at(db, k * 2048), kPv, add || k > 0);
#pragma unroll
        for (uint32_t k = 4 * part; k < 4 * part + 4; ++k)
          mma_ts(tmem + o_col(half), tmem + p_col(half, 16 * k), desc_at(db, k * 2048), kPv, add || k > 0);
        mma_commit(smem_u32(&sh.pv_done[half][part]));
      }
      __syncwarp();
    }
    return true;
  };
  // Key tiles [0, plain) of L of a kRowsApart tile, by one lane.  before[s][part]:
  // uses of the weights' barriers so far, by their parity.
  auto steady = [&](uint32_t L, uint32_t plain, uint32_t item0, const uint32_t (&before)[2][2]) {
    const uint64_t k_base = tile_desc(ring, 16), v_base = tile_desc(ring, kSlabBytes);
    const uint64_t q_desc[2] = {tile_desc(q_smem, 16), tile_desc(q_smem + Sh::kTile, 16)};
#pragma unroll 1
    for (uint32_t j = 0; j < plain; ++j) {
      const uint32_t v_item = item0 + 2 * j + 1, k_next = v_item + 1;
      const uint32_t v_at = v_item % Sh::kRing, k_at = k_next % Sh::kRing;
      const uint64_t v_desc = desc_at(v_base, v_at * Sh::kTile), k_desc = desc_at(k_base, k_at * Sh::kTile);
      const bool more = j + 1 < L;
      if (!mbar_wait_lane(smem_u32(&sh.full[v_at]), (v_item / Sh::kRing) & 1, a.limit)) return false;
#pragma unroll
      for (uint32_t s = 0; s < 2; ++s) {
#pragma unroll
        for (uint32_t part = 0; part < 2; ++part) {
          if (!mbar_wait_lane(smem_u32(&sh.p_full[s][part]), (before[s][part] + j) & 1, a.limit)) return false;
          tc_fence_after();
#pragma unroll
          for (uint32_t k = 4 * part; k < 4 * part + 4; ++k)
            mma_ts(tmem + o_col(s), tmem + p_col(s, 16 * k), desc_at(v_desc, k * 2048), kPv, j > 0 || k > 0);
          mma_commit(smem_u32(&sh.pv_done[s][part]));
        }
        if (s == 1) release(v_at);
        if (more) {
          if (s == 0 && !mbar_wait_lane(smem_u32(&sh.full[k_at]), (k_next / Sh::kRing) & 1, a.limit)) return false;
          // in order after the product above, which reads the weights that these scores overwrite
          mma_ss<false>(tmem + s_col(s), q_desc[s], k_desc, kQk);
#pragma unroll
          for (uint32_t k = 1; k < NSLAB * 4; ++k) {
            const uint32_t off = (k / 4) * kSlabBytes + (k % 4) * 32;
            if (k < steps) mma_ss<true>(tmem + s_col(s), desc_at(q_desc[s], off), desc_at(k_desc, off), kQk);
          }
          mma_commit(smem_u32(&sh.s_full[s]));
          if (j + 2 == L) mma_commit(smem_u32(&sh.q_empty[s]));
        }
      }
      if (more) release(k_at);
    }
    return true;
  };
  Walk w;
  for (bool more = w.begin(a); more; more = w.next(a)) {
    const int mode = KIND == kFew ? kColumnsApart : w.mode(a);
    const uint32_t L = w.kv1 - w.kv0;
    // slots that hold no token may hold NaN: zero their values (their weights are zero)
    auto clear_tail = [&](uint32_t j, uint32_t v_item) {
      const uint64_t first = (uint64_t)(w.kv0 + j) * kKeys;
      if (first + kKeys <= w.n) return;
      const uint32_t have = w.n > first ? (uint32_t)(w.n - first) : 0;
      for (uint32_t i = have * (NSLAB * 8) + lane; i < kKeys * NSLAB * 8; i += 32) {
        const uint32_t row = i / (NSLAB * 8), c = i % (NSLAB * 8);
        const uint32_t at = tile_at(v_item) + (c / 8) * kSlabBytes + row * 128 + (c % 8) * 16;
        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0u) : "memory");
      }
      fence_async_shared();
      __syncwarp();
    };
    if (!mbar_wait(smem_u32(&sh.q_full[0]), used[0]++ & 1, a.limit) || !full(item)) return false;
    tc_fence_after();
    scores(0, 0, item);
    if (mode == kRowsApart) {
      if (!mbar_wait(smem_u32(&sh.q_full[1]), used[1]++ & 1, a.limit)) return false;
      tc_fence_after();
      scores(1, 1, item);
      free_tile(item);
      if (L == 1) {
        commit(sh.q_empty[0]);
        commit(sh.q_empty[1]);
      }
      // All tiles but one that has slots to clear: one lane by itself, as the
      // tensor cores wait whenever their queue runs dry between two products
      // (with the warp's votes in between, a unit took 3,030 cycles for 2,048 of
      // products).
      const uint32_t plain = (uint64_t)w.kv1 * kKeys > w.n ? L - 1 : L;
      bool ok = true;
      if (elect_lane()) ok = steady(L, plain, item, weights);
      if (!__all_sync(kFull, ok)) return false;
      for (uint32_t s = 0; s < 2; ++s)
        for (uint32_t part = 0; part < 2; ++part) weights[s][part] += plain;
      for (uint32_t j = plain; j < L; ++j) {
        const uint32_t v_item = item + 2 * j + 1, k_next = v_item + 1;
        if (!full(v_item)) return false;
        clear_tail(j, v_item);
        for (uint32_t s = 0; s < 2; ++s) {
          if (!values(s, v_item, j > 0, true)) return false;
          if (s == 1) free_tile(v_item);
          if (j + 1 < L) {
            if (s == 0 && !full(k_next)) return false;
            // in order after the product above, which reads the weights that these scores overwrite
            scores(s, s, k_next);
            if (j + 2 == L) commit(sh.q_empty[s]);
          }
        }
        if (j + 1 < L) free_tile(k_next);
      }
    } else {
      free_tile(item);
      if (L > 1) {
        if (!full(item + 2)) return false;
        tc_fence_after();
        scores(1, 0, item + 2);
        free_tile(item + 2);
      }
      if (L <= 2) commit(sh.q_empty[0]);
      for (uint32_t j = 0; j < L; ++j) {
        const uint32_t v_item = item + 2 * j + 1, k_next = item + 2 * j + 4;
        if (!full(v_item)) return false;
        clear_tail(j, v_item);
        if (!values(j & 1, v_item, j > 1, mode != kColumnsApart)) return false;
        free_tile(v_item);
        if (j + 2 < L) {
          if (!full(k_next)) return false;
          scores(j & 1, 0, k_next);
          free_tile(k_next);
          if (j + 3 == L) commit(sh.q_empty[0]);
        }
      }
    }
    item += 2 * L;
  }
  return true;
}

// Queries by tensor copies, a tile ahead of the products.
template <int NSLAB, int KIND>
__device__ __forceinline__ bool query_role(const AttnArgs& a, TileShared& sh, const CUtensorMap* mq,
                                           const CUtensorMap* mq32, uint32_t q_smem, uint32_t (&loads)[2]) {
  using Sh = TileShape<NSLAB, KIND>;
  const uint32_t lane = threadIdx.x & 31;
  if (a.withhold) return true;
  Walk w;
  for (bool more = w.begin(a); more; more = w.next(a)) {
    const int mode = KIND == kFew ? kColumnsApart : w.mode(a);
    const int tok = (int)(w.tok0 + w.token0(a));
    for (uint32_t s = 0; s < (mode == kRowsApart ? 2u : 1u); ++s) {
      if (loads[s] && !mbar_wait(smem_u32(&sh.q_empty[s]), (loads[s] - 1) & 1, a.limit)) return false;
      ++loads[s];
      const uint32_t bar = smem_u32(&sh.q_full[s]), dst = q_smem + s * Sh::kTile;
      if (lane == 0) sh.loads[s] = loads[s];
      if (lane == 0 && mode != kColumnsApart) {
        mbar_expect(bar, NSLAB * a.tq * a.G * 128);
#pragma unroll
        for (int c = 0; c < NSLAB; ++c) tma_load_4d(dst + c * kSlabBytes, mq, bar, 64 * c, 0, (int)w.h, tok + (int)(s * a.tq));
      } else if (lane == 0) {
        mbar_expect(bar, 4 * NSLAB * a.tq32 * a.G * 128);
        for (int x = 0; x < 4; ++x)
#pragma unroll
          for (int c = 0; c < NSLAB; ++c) tma_load_4d(dst + c * kSlabBytes + x * 4096, mq32, bar, 64 * c, 0, (int)w.h, tok);
      }
      __syncwarp();
    }
  }
  return true;
}

// Keys and values by tensor copies, a warp for each: a copy a stretch of `box` slots (a divisor
// of the page size and of the tile) and slab.  Stretches at or past the
// request's end and pages that the cache does not have read as zeros: their
// page coordinate is n_pages, which is out of range.
template <int NSLAB, int KIND>
__device__ __forceinline__ bool copy_role(const AttnArgs& a, TileShared& sh, const CUtensorMap* map,
                                          uint32_t ring, uint32_t kv) {
  using Sh = TileShape<NSLAB, KIND>;
  const uint32_t lane = threadIdx.x & 31, boxes = kKeys / a.box;
  Walk w;
  if (!w.begin(a)) return true;
  // the page of the lane's stretch of key tile j, asked for a tile ahead
  uint32_t issued = 0, j = w.kv0, id = 0, slot = 0, head = 0;
  bool in = false;
  auto ask = [&] {
    const uint32_t key = j * kKeys + lane * a.box, at = key / a.kv.B;
    in = lane < boxes && key < w.n;
    slot = key - at * a.kv.B;
    head = w.h;
    id = in ? __ldg(a.kv.page_ids + w.page0 + at) : 0;
  };
  ask();
  for (bool more = true; more;) {
    int page = (int)a.kv.n_pages;
    if (in && id < a.kv.n_pages) page = (int)id;
    else if (in) report(a.status, PTC_ERR_INVALID_ARG);
    const int s0 = in ? (int)slot : 0, h0 = (int)head;
    if (++j == w.kv1) {
      more = w.next(a);
      j = w.kv0;
    }
    if (more) ask();
    const uint32_t item = 2 * issued++ + kv, at = item % Sh::kRing;
    if (item >= Sh::kRing && !mbar_wait(smem_u32(&sh.empty[at]), (item / Sh::kRing - 1) & 1, a.limit)) return false;
    const uint32_t bar = smem_u32(&sh.full[at]), dst = ring + at * Sh::kTile + lane * a.box * 128;
    if (lane == 0) {
      sh.issued[kv] = issued;
      mbar_expect(bar, Sh::kTile);
    }
    __syncwarp();
    if (lane < boxes)
#pragma unroll
      for (int s = 0; s < NSLAB; ++s) tma_load_4d(dst + s * kSlabBytes, map, bar, 64 * s, s0, h0, page);
  }
  return true;
}

// The same for page sizes that are no multiple of 8 (a swizzled tile takes
// copies of whole groups of 8 rows): 64 threads copy 16 bytes each.  Ten times
// slower, and bound by these threads' own steps, two divisions and a page id for
// every 16 bytes: with pages of 12, 64 single tokens (0.89 GB) take 1.56 ms for
// 0.16 with pages of 16, 4,096 tokens at 32K 10.8 ms for 1.22.
template <int NSLAB, int KIND>
__device__ __forceinline__ bool gather_role(const AttnArgs& a, TileShared& sh, uint32_t ring) {
  using Sh = TileShape<NSLAB, KIND>;
  const uint32_t tid = (threadIdx.x & 31) + (threadIdx.x >= 352 ? 32 : 0);
  uint32_t issued = 0, landed = 0;
  auto land = [&](uint32_t upto) {
    fence_async_shared();
    for (; landed < upto; ++landed) mbar_arrive(smem_u32(&sh.full[landed % Sh::kRing]));
  };
  Walk w;
  for (bool more = w.begin(a); more; more = w.next(a)) {
    const uint32_t* ids = a.kv.page_ids + w.page0;
    for (uint32_t j = w.kv0; j < w.kv1; ++j)
      for (int kv = 0; kv < 2; ++kv) {
        const uint32_t at = issued % Sh::kRing;
        if (issued >= Sh::kRing && !mbar_wait(smem_u32(&sh.empty[at]), (issued / Sh::kRing - 1) & 1, a.limit)) {
          cp_async_wait<0>();
          return false;
        }
        const char* src = kv == 0 ? a.kv.k : a.kv.v;
        const int64_t sp = kv == 0 ? a.kv.ks_page : a.kv.vs_page, ss = kv == 0 ? a.kv.ks_slot : a.kv.vs_slot;
        const int64_t head = w.h * (kv == 0 ? a.kv.ks_head : a.kv.vs_head);
        for (uint32_t i = tid; i < kKeys * NSLAB * 8; i += 64) {
          const uint32_t row = i / (NSLAB * 8), c = i % (NSLAB * 8);
          const uint32_t key = j * kKeys + row;
          bool in = key < w.n && c * 8 < a.kv.D;
          const char* p = src;
          if (in) {
            const uint32_t id = __ldg(ids + key / a.kv.B);
            in = id < a.kv.n_pages;
            if (in) p = src + 2 * (id * sp + head + (int64_t)(key % a.kv.B) * ss + c * 8);
            else report(a.status, PTC_ERR_INVALID_ARG);
          }
          cp_async16(ring + at * Sh::kTile + (c / 8) * kSlabBytes + row * 128 + (((c % 8) ^ (row & 7)) * 16), p, in);
        }
        cp_async_commit();
        ++issued;
        cp_async_wait<2>();
        if (issued > 2) land(issued - 2);
      }
  }
  cp_async_wait<0>();
  land(issued);
  return true;
}

// Keys and values out of pages of 4 bits, by four warps in place of the two of the
// tensor copies.  A warp copies 32 rows of a tile into a ring of its own (16 bytes a
// lane, a tile or two ahead), and takes its rows' codes to 16-bit numbers in the
// ring of tiles, swizzled as the products want them: four (two) lanes a row, 32
// channels each, three instructions and half a store for two values.  Slots of no
// token, or of a page that the cache does not have, are zeros.
//
// Bounds.  Shared memory: the products read 192 KB a pair of tiles, these warps write
// 64, and 20 of codes go in and out, 2,520 cycles at 128 bytes a cycle of the 3,240
// that a pair takes (without any of these warps' traffic 2,700, as over 16-bit pages;
// without their arithmetic no less).  Loading the codes into registers instead took
// 1.68 to 3.19 ms for the 1.47 of 4,096 tokens at 32K.
template <typename T, int NSLAB>
__device__ __forceinline__ bool quant_role(const AttnArgs& a, TileShared& sh, uint32_t ring, uint32_t tiles4) {
  using Sh = TileShape<NSLAB, kFour>;
  constexpr uint32_t kLanes = 2 * NSLAB, kSteps = kLanes;  // lanes of a row, rows of a lane
  constexpr uint32_t kCodes = 32 * NSLAB;                               // bytes of a row's codes
  constexpr uint32_t kMine = 32 * Sh::kRow4;                            // bytes of the warp's part of a tile
  const uint32_t lane = threadIdx.x & 31, row0 = 32 * (threadIdx.x / 32 - 12);
  const uint32_t mine = tiles4 + row0 / 32 * Sh::kRing4 * kMine;
  // copies: every lane finds a row; item 2 j + 1, a tile's values, follows item 2 j, its keys.
  // The walk waits in shared memory from one part to the next: 72 registers are few.
  Walk& rest = reinterpret_cast<Walk*>(&sh + 1)[row0 / 32];
  bool more, values = false;
  uint32_t j = 0, end = 0, n = 0, id = kNone, slot = 0, rows = 0, issued = 0;
  const char *kb = nullptr, *vb = nullptr, *k = nullptr, *v = nullptr;  // the head's rows of page 0; the lane's rows
  const uint32_t* ids = nullptr;
  auto part = [&](const Walk& w) {
    j = w.kv0;
    end = w.kv1;
    n = w.n;
    ids = a.kv.page_ids + w.page0;
    kb = a.kv.k + w.h * a.kv.ks_head;
    vb = a.kv.v + w.h * a.kv.vs_head;
    __syncwarp();
    if (lane == 0) rest = w;
    __syncwarp();
  };
  auto key_of = [&] { return j * kKeys + row0 + lane; };
  auto ask = [&] {
    const uint32_t key = key_of(), at = a.kv.B == 1 ? key : __umulhi(key, a.div_mul) >> a.div_shift;
    slot = key - at * a.kv.B;
    id = key < n ? __ldg(ids + at) : kNone;
  };
  {
    Walk w;
    more = w.begin(a);
    if (more) {
      part(w);
      ask();
    }
  }
  auto issue = [&] {
    if (!values && more) {
      const bool on = id < a.kv.n_pages;
      if (!on && key_of() < n) report(a.status, PTC_ERR_INVALID_ARG);  // (any id: a list may hold kNone)
      rows = __ballot_sync(kFull, on);
      const uint32_t page = on ? id : 0, s = on ? slot : 0;
      k = kb + page * a.kv.ks_page + s * a.kv.ks_slot;
      v = vb + page * a.kv.vs_page + s * a.kv.vs_slot;
      if (++j == end) {
        Walk w = rest;
        more = w.next(a);
        if (more) part(w);
      }
      if (more) ask();
    } else if (!values) {
      cp_async_commit();
      return;
    }
    // all rows' codes, then all rows' scales and bases
    const uint32_t dst = mine + issued % Sh::kRing4 * kMine + 16 * lane;
    const char* from = values ? v : k;
#pragma unroll
    for (uint32_t i = 0; i < kSteps; ++i) {
      const uint32_t row = 32 / kLanes * i + lane / kLanes;
      const char* x = reinterpret_cast<const char*>(__shfl_sync(kFull, reinterpret_cast<uint64_t>(from), row));
      cp_async16(dst + 512 * i, x + 16 * (lane % kLanes), rows >> row & 1);
    }
    cp_async16(dst + 32 * kCodes, from + kCodes, rows >> lane & 1);
    cp_async_commit();
    ++issued;
    values = !values;
  };
#pragma unroll 1
  for (uint32_t i = 0; i + 1 < Sh::kRing4; ++i) issue();
  // The lane's rows are first, first + 32 / kLanes and so on.  (The second slab's
  // rows are two off: the loads and the stores of eight lanes meet no bank twice.)
  const uint32_t group = lane % kLanes, first = (lane / kLanes) ^ (group & 2);
  const uint32_t codes_at = mine + first * kCodes + 16 * group, pars_at = mine + 32 * kCodes + 16 * first + 4 * group;
  const uint32_t piece0 = (4 * (group & 1)) ^ (first & 7);
  const uint32_t tile_at = ring + group / 2 * kSlabBytes + (row0 + first) * 128;
  for (uint32_t item = 0; item < issued; ++item) {
    cp_async_wait<Sh::kRing4 - 2>();
    __syncwarp();  // the rows are there for all lanes, and all are through with the tile before
    issue();
    const uint32_t at = item % Sh::kRing, src = item % Sh::kRing4 * kMine;
    uint32_t c[kSteps][4], par[kSteps];
#pragma unroll
    for (uint32_t i = 0; i < kSteps; ++i) {
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(c[i][0]), "=r"(c[i][1]), "=r"(c[i][2]), "=r"(c[i][3])
                   : "r"(codes_at + src + 512 * i)
                   : "memory");
      asm volatile("ld.shared.b32 %0, [%1];" : "=r"(par[i]) : "r"(pars_at + src + 512 / kLanes * i) : "memory");
    }
    if (item >= Sh::kRing && !mbar_wait(smem_u32(&sh.empty[at]), (item / Sh::kRing - 1) & 1, a.limit)) {
      cp_async_wait<0>();
      return false;
    }
    const uint32_t to = tile_at + at * Sh::kTile;
#pragma unroll
    for (uint32_t i = 0; i < kSteps; ++i) {
      const uint32_t s = both_low(par[i]), b = both_high(par[i]);
#pragma unroll
      for (uint32_t x = 0; x < 4; ++x)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + 16 * (piece0 ^ x) + 4096 / kLanes * i),
                     "r"(fma16x2<T>(pair4<T>(c[i][x], 0), s, b)), "r"(fma16x2<T>(pair4<T>(c[i][x], 1), s, b)),
                     "r"(fma16x2<T>(pair4<T>(c[i][x], 2), s, b)), "r"(fma16x2<T>(pair4<T>(c[i][x], 3), s, b))
                     : "memory");
    }
    fence_async_shared();
    mbar_arrive_warp(smem_u32(&sh.full[at]));
  }
  cp_async_wait<0>();
  return true;
}

// Where a role has given up: all tensor copies that were issued land before the
// CTA ends, also those of a role that has issued all of its own.  A place of the
// ring was taken again only after its products, so its last copy is the one
// that may be in flight.  By one warp.
template <uint32_t RING>
__device__ __noinline__ void land_copies(TileShared& sh) {
  for (uint32_t at = 0; at < RING; ++at) {
    uint32_t next = 0;  // the place's last copy, and one
    for (uint32_t kv = 0; kv < 2; ++kv)
      for (uint32_t i = sh.issued[kv], k = 0; i > 0 && k < RING; --i, ++k) {
        const uint32_t item = 2 * (i - 1) + kv;
        if (item % RING != at) continue;
        if (item + 1 > next) next = item + 1;
        break;
      }
    if (next) (void)mbar_wait(smem_u32(&sh.full[at]), ((next - 1) / RING) & 1);
  }
  for (int s = 0; s < 2; ++s)
    if (sh.loads[s]) (void)mbar_wait(smem_u32(&sh.q_full[s]), (sh.loads[s] - 1) & 1);
}

template <typename T, int NSLAB, bool TMA, int KIND>
__global__ void __launch_bounds__(TileShape<NSLAB, KIND>::kThreads, 1)
    k_attn_tiles(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv,
                 const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mq32, const AttnArgs a) {
  using Sh = TileShape<NSLAB, KIND>;
  extern __shared__ __align__(1024) char smem_raw[];
  TileShared& sh = *reinterpret_cast<TileShared*>(smem_raw + Sh::kRest);
  const uint32_t q_smem = smem_u32(smem_raw), ring = q_smem + Sh::kQueries * Sh::kTile;
  const uint32_t warp = threadIdx.x >> 5;
  if (q_smem & 1023) {  // swizzled tiles start at whole groups of 8 rows
    if (threadIdx.x == 0) report(a.status, PTC_ERR_CUDA);
    return;
  }
  if (threadIdx.x == 0) {
    for (uint32_t i = 0; i < Sh::kRing; ++i) {
      mbar_init(smem_u32(&sh.full[i]), KIND == kFour ? 4 : TMA ? 1 : 64);
      mbar_init(smem_u32(&sh.empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sh.q_full[i]), 1);
      mbar_init(smem_u32(&sh.q_empty[i]), 1);
      mbar_init(smem_u32(&sh.s_full[i]), 1);
      for (int part = 0; part < 2; ++part) {
        mbar_init(smem_u32(&sh.p_full[i][part]), 4);
        mbar_init(smem_u32(&sh.pv_done[i][part]), 1);
      }
    }
    mbar_init(smem_u32(&sh.drain), 1);
    fence_mbar_init();
    for (int i = 0; i < 2; ++i) sh.issued[i] = sh.loads[i] = 0;
  }
  if (warp == 8) tmem_alloc(smem_u32(&sh.tmem), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  grid_dep_sync();
  const bool go = a.plan->ok != 0;
  bool fine = true;
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Sh::kSoftmax));
    if (go) fine = softmax_role<T, NSLAB, KIND>(a, sh, smem_raw + Sh::kRest - kStage, warp / 4);
  } else if (KIND == kFour && warp >= 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kQuantRegs4));
    if (go) fine = quant_role<T, NSLAB>(a, sh, ring, ring + Sh::kRing * Sh::kTile);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Sh::kOther));
    // (declared inside query_role, the registers fall so that the softmax spills: 1.23 -> 1.6 ms for 4,096 tokens at 32K)
    uint32_t loads[2] = {0, 0};
    if (!go) {
    } else if (warp == 8) {
      fine = product_role<T, NSLAB, KIND>(a, sh, q_smem, ring);
      // every product and every arrival it owes is done before the CTA ends
      if (elect_lane()) mma_commit(smem_u32(&sh.drain));
      __syncwarp();
      fine &= mbar_wait(smem_u32(&sh.drain), 0);
    } else if (warp == 10) {
      fine = query_role<NSLAB, KIND>(a, sh, &mq, &mq32, q_smem, loads);
    } else if (KIND == kFour) {
    } else if (!TMA) {
      fine = gather_role<NSLAB, KIND>(a, sh, ring);
    } else {
      fine = copy_role<NSLAB, KIND>(a, sh, warp == 9 ? &mk : &mv, ring, warp == 9 ? 0 : 1);
    }
  }
  if (!fine) report(a.status, PTC_ERR_TIMEOUT);
  tc_fence_before();
  if (__syncthreads_or(!fine)) {
    if (warp == 9) land_copies<Sh::kRing>(sh);
    __syncthreads();
  }
  tc_fence_after();
  if (warp == 8) tmem_free(sh.tmem, 512);
}

}  // namespace
}  // namespace ptc
