// Attention of new tokens over paged keys and values (ptc_paged_attention).
#include <cmath>

#include "ptc_kv.cuh"
#include "ptc_tc.cuh"

namespace ptc {
namespace {

// Rows of a query tile, keys of a key tile.  The G query heads of a key head
// are packed as rows of one matrix, row = token * G + head, so that a key tile
// is read once for all of them.
constexpr uint32_t kRows = 256, kKeys = 128;
constexpr uint32_t kMaxCtas = 512;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Where a CTA of the tile kernel starts: its first unit, and what that is.
struct CtaStart {
  uint64_t u;
  uint32_t r, h, qt, kv;
};

// What k_attn_plan leaves for the kernels after it.  The work of a call is a
// row of units: for every request, key head and query tile, its key tiles.
// CTA c of C takes the units [U c / C, U (c + 1) / C).
struct AttnPlan {
  uint32_t ok, pad;
  uint64_t units;
  CtaStart start[kMaxCtas];
};

struct AttnArgs {
  KvView kv;
  const char* q;
  int64_t q_tok, q_head;
  const uint64_t* tok_off;
  uint64_t n_tok;
  uint32_t n_q_heads, G, max_q_len;
  float scale;
  char* out;
  float* lse;
  const float* mass_in;
  float* mass_out;
  uint64_t mass_stride;
  AttnPlan* plan;
  uint64_t* unit_off;  // n_req + 1
  float* part;         // unnormalised rows of split tiles: [2 * ctas][kRows][D]
  float2* part_ml;     // their maxima (in powers of two) and sums
  uint32_t ctas, box;  // box: rows of a tensor copy
  uint32_t* status;
};

// Key tiles that query tile qt of a request sees, at least one.
__device__ __forceinline__ uint32_t key_tiles(uint32_t m, uint32_t n, uint32_t G, uint32_t qt) {
  const uint32_t rows = m * G, end = (qt + 1) * kRows < rows ? (qt + 1) * kRows : rows;
  const int64_t sees = (int64_t)n - m + (end - 1) / G + 1;
  return sees <= (int64_t)kKeys ? 1u : (uint32_t)((sees + kKeys - 1) / kKeys);
}

// req_search over offsets that this kernel has written itself.
__device__ __forceinline__ uint32_t unit_search(const uint64_t* off, uint32_t lo, uint32_t hi, uint64_t u) {
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo + 1) / 2;
    if (ld_relaxed_u64(off + mid) <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// The requests' share of the units, and every CTA's start.  One CTA: the
// lists are a few KB, and a second pass over them would cost a launch.
constexpr int kPlanThreads = 1024;
__global__ void __launch_bounds__(kPlanThreads) k_attn_plan(AttnArgs a) {
  asm volatile("griddepcontrol.launch_dependents;");
  grid_dep_sync();
  __shared__ uint64_t s_warp[32];
  const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, R = a.kv.n_req, G = a.G;
  bool bad = tid == 0 && (a.tok_off[0] != 0 || a.tok_off[R] != a.n_tok);
  uint64_t carry = 0;
  for (uint32_t r0 = 0; r0 < R; r0 += kPlanThreads) {
    const uint32_t r = r0 + tid;
    uint32_t m = 0, n = 0;
    if (r < R) {
      const uint64_t lo = a.tok_off[r], hi = a.tok_off[r + 1];
      n = a.kv.kv_len[r];
      const bool wrong = lo > hi || hi > a.n_tok || hi - lo > a.max_q_len || !pages_hold(a.kv, r, n);
      bad |= wrong;
      m = wrong ? 0 : (uint32_t)(hi - lo);
    }
    const uint32_t tiles = (m * G + kRows - 1) / kRows;
    uint64_t mine = 0;
    if (tiles <= 2)
      for (uint32_t qt = 0; qt < tiles; ++qt) mine += key_tiles(m, n, G, qt);
    // requests of many tiles: a warp adds one up
    for (uint32_t todo = __ballot_sync(kFull, tiles > 2); todo; todo &= todo - 1) {
      const int src = __ffs(todo) - 1;
      const uint32_t mm = __shfl_sync(kFull, m, src), nn = __shfl_sync(kFull, n, src),
                     tt = __shfl_sync(kFull, tiles, src);
      uint64_t sum = 0;
      for (uint32_t qt = lane; qt < tt; qt += 32) sum += key_tiles(mm, nn, G, qt);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
      if (lane == (uint32_t)src) mine = sum;
    }
    mine *= a.kv.H;
    uint64_t incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(kFull, incl, o);
      if (lane >= (uint32_t)o) incl += y;
    }
    if (lane == 31) s_warp[warp] = incl;
    __syncthreads();
    uint64_t before = carry + incl - mine, all = carry;
    for (uint32_t w = 0; w < 32; ++w) {
      if (w < warp) before += s_warp[w];
      all += s_warp[w];
    }
    if (r < R) a.unit_off[r] = before;
    carry = all;
    __syncthreads();
  }
  bad = __syncthreads_or(bad);
  if (tid == 0) {
    a.unit_off[R] = carry;
    a.plan->ok = !bad;
    a.plan->units = carry;
    if (bad) report(a.status, PTC_ERR_INVALID_ARG);
  }
  if (bad) return;
  __syncthreads();
  for (uint32_t c = warp; c < a.ctas; c += 32) {
    const uint64_t u = carry * c / a.ctas;
    CtaStart s{u, 0, 0, 0, 0};
    if (u < carry) {
      s.r = unit_search(a.unit_off, 0, R - 1, u);
      const uint32_t m = (uint32_t)(a.tok_off[s.r + 1] - a.tok_off[s.r]), n = a.kv.kv_len[s.r];
      const uint64_t at = ld_relaxed_u64(a.unit_off + s.r), in = u - at;
      const uint64_t head = (ld_relaxed_u64(a.unit_off + s.r + 1) - at) / a.kv.H;
      s.h = (uint32_t)(in / head);
      uint64_t rest = in % head;
      const uint32_t tiles = (m * G + kRows - 1) / kRows;
      for (uint32_t q0 = 0; q0 < tiles; q0 += 32) {
        const uint32_t k = q0 + lane < tiles ? key_tiles(m, n, G, q0 + lane) : 0;
        uint32_t incl = k;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t y = __shfl_up_sync(kFull, incl, o);
          if (lane >= (uint32_t)o) incl += y;
        }
        const uint32_t here = __ballot_sync(kFull, rest < incl);
        if (here) {
          const int src = __ffs(here) - 1;
          s.qt = q0 + src;
          s.kv = (uint32_t)rest - __shfl_sync(kFull, incl - k, src);
          break;
        }
        rest -= __shfl_sync(kFull, incl, 31);
      }
    }
    if (lane == 0) a.plan->start[c] = s;
  }
}

// The query tiles that a CTA has a part in, in order, with the part.
struct Walk {
  uint64_t left, tok0, page0;
  uint32_t r, h, qt, kv0, kv1, nkv;  // key tiles [kv0, kv1) of nkv
  uint32_t m, n, rows, pages;
  __device__ __forceinline__ void request(const AttnArgs& a) {
    tok0 = a.tok_off[r];
    m = (uint32_t)(a.tok_off[r + 1] - tok0);
    n = a.kv.kv_len[r];
    rows = m * a.G;
    page0 = a.kv.page_off[r];
    pages = (uint32_t)(a.kv.page_off[r + 1] - page0);
  }
  __device__ __forceinline__ void part(const AttnArgs& a) {
    nkv = key_tiles(m, n, a.G, qt);
    kv1 = nkv - kv0 > left ? kv0 + (uint32_t)left : nkv;
  }
  // False if the CTA has nothing to do.
  __device__ __forceinline__ bool begin(const AttnArgs& a) {
    const uint64_t U = a.plan->units, c = blockIdx.x;
    const CtaStart s = a.plan->start[c];
    left = U * (c + 1) / a.ctas - s.u;
    if (left == 0) return false;
    r = s.r;
    h = s.h;
    qt = s.qt;
    kv0 = s.kv;
    request(a);
    part(a);
    return true;
  }
  __device__ __forceinline__ bool next(const AttnArgs& a) {
    left -= kv1 - kv0;
    if (left == 0) return false;
    kv0 = 0;
    if (++qt * kRows >= rows) {
      qt = 0;
      if (++h == a.kv.H) {
        h = 0;
        do {
          if (++r == a.kv.n_req) return false;
          request(a);
        } while (m == 0);
      }
    }
    part(a);
    return true;
  }
};

// Two 32-bit floats rounded to the cache's type, the first in the low half.
// Attention weights of bf16 caches are rounded as they are.  Those of fp16
// caches are scaled by 2^7 first: a weight far below the running maximum would
// otherwise fall among fp16's subnormals (below 2^-14) and a long row of small
// weights would be lost; with the lazy maximum's 2^8 the largest is 2^15.
template <typename T>
struct Weights;
template <>
struct Weights<__nv_bfloat16> {
  static constexpr bool kBf16 = true;
  static constexpr float kShift = 0.f;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
};
template <>
struct Weights<__half> {
  static constexpr bool kBf16 = false;
  static constexpr float kShift = 7.f;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 x = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
};

// ------------------------------------------------------------------ the tile kernel
// One CTA an SM walks its units.  Warps 0-3 and 4-7 are the softmax of the
// query tile's rows 0-127 and 128-255, warp 8 issues the products, warp 9 (with
// tensor copies; warps 9-11 without) loads keys and values into a ring of
// tiles.  For key tile j:
//   scores   S = Q K_j^T     128 x 128 sums in tensor memory
//   softmax  one thread a row: running maximum and sum in 32 bits; weights
//            exp2(s - max), rounded to 16 bits, over the scores' columns
//   values   O += P V_j      P from tensor memory, O stays there
// The two halves alternate: while one is in its softmax, the tensor cores work
// for the other.  O is rescaled only when a row's maximum has grown by more
// than a factor of 2^8 since the last time (weights up to 2^8 are as exact as
// those up to 1), which after the first tiles hardly happens.
constexpr int kTileThreads = 384;
constexpr int kSlabBytes = 128 * 128;  // 128 rows of 64 columns

template <int NSLAB>
struct TileShape {
  static constexpr int kTile = NSLAB * kSlabBytes;
  static constexpr int kRing = NSLAB == 2 ? 5 : 8;
  static constexpr int kSmem = 2 * kTile + kRing * kTile + 1024;
};

struct TileShared {
  uint64_t full[8], empty[8], q_full[2], s_full[2], p_full[2], pv_done[2], drain;
  uint32_t tmem, abort;
};

// Tensor memory columns: scores (and weights) of both halves, then their sums.
__device__ __forceinline__ uint32_t s_col(uint32_t half) { return half * 128; }
__device__ __forceinline__ uint32_t o_col(uint32_t half) { return 256 + half * 128; }

template <typename T, int NSLAB>
__device__ __forceinline__ bool softmax_role(const AttnArgs& a, TileShared& sh, uint32_t q_smem, uint32_t half) {
  using W = Weights<T>;
  const uint32_t tid = threadIdx.x & 127;
  const uint32_t tmem = sh.tmem + ((tid & ~31u) << 16);
  const uint32_t s_at = tmem + s_col(half), o_at = tmem + o_col(half);
  const uint32_t bar_s = smem_u32(&sh.s_full[half]), bar_p = smem_u32(&sh.p_full[half]),
                 bar_o = smem_u32(&sh.pv_done[half]), bar_q = smem_u32(&sh.q_full[half]);
  const float sl2 = a.scale * kLog2e, slack = fminf(8.f / sl2, 1e38f);
  const uint32_t D = a.kv.D;
  const uint32_t qs = q_smem + half * TileShape<NSLAB>::kTile;
  uint32_t done = 0;  // key tiles of this half so far
  Walk w;
  for (bool more = w.begin(a); more; more = w.next(a)) {
    const uint32_t row0 = w.qt * kRows + half * 128;
    if (row0 >= w.rows) continue;
    // the query rows, zero beyond the request and beyond head_dim
    const char* q = a.q + 2 * ((int64_t)w.tok0 * a.q_tok + (int64_t)w.h * a.G * a.q_head);
#pragma unroll 8
    for (uint32_t i = 0; i < NSLAB * 8; ++i) {
      const uint32_t id = i * 128 + tid, row = id / (NSLAB * 8), c = id % (NSLAB * 8);
      uint4 x = make_uint4(0, 0, 0, 0);
      if (row0 + row < w.rows && c * 8 < D) {
        const uint32_t t = (row0 + row) / a.G, g = (row0 + row) % a.G;
        x = *reinterpret_cast<const uint4*>(q + 2 * ((int64_t)t * a.q_tok + (int64_t)g * a.q_head + c * 8));
      }
      const uint32_t at = qs + (c / 8) * kSlabBytes + row * 128 + (((c % 8) ^ (row & 7)) * 16);
      asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
    }
    fence_async_shared();
    mbar_arrive(bar_q);

    const uint32_t row = row0 + tid;
    const bool valid = row < w.rows;
    const uint32_t t = row / a.G, g = row % a.G;
    const bool active = __any_sync(kFull, valid);
    int64_t left = valid ? (int64_t)w.n - w.m + t + 1 - (int64_t)w.kv0 * kKeys : 0;  // keys from this tile on that the row sees
    float top = -INFINITY, l = 0.f;
    for (uint32_t j = w.kv0; j < w.kv1; ++j, ++done, left -= kKeys) {
      if (!mbar_wait(bar_s, done & 1)) return false;
      tc_fence_after();
      if (active) {
        const int see = left >= (int64_t)kKeys ? (int)kKeys : left > 0 ? (int)left : 0;
        const bool masked = __any_sync(kFull, see < (int)kKeys);
        float mx = -INFINITY;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t x[32];
          tmem_ld32(x, s_at + 32 * c);
          tmem_wait_ld();
          if (masked) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (32 * c + i >= see) x[i] = 0xFF800000u;
          }
#pragma unroll
          for (int i = 0; i < 32; ++i) mx = fmaxf(mx, __uint_as_float(x[i]));
        }
        if (__any_sync(kFull, mx > top + slack)) {
          const float nt = fmaxf(top, mx);
          const float f = top == -INFINITY ? 0.f : exp2_approx((top - nt) * sl2);
          l *= f;
          top = nt;
          if (j > w.kv0) {
            if (!mbar_wait(bar_o, (done - 1) & 1)) return false;
            tc_fence_after();
#pragma unroll
            for (int c = 0; c < NSLAB * 2; ++c) {
              uint32_t x[32];
              tmem_ld32(x, o_at + 32 * c);
              tmem_wait_ld();
#pragma unroll
              for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * f);
              tmem_st32(o_at + 32 * c, x);
            }
          }
        }
        const float sub = (top == -INFINITY ? 0.f : top * sl2) - W::kShift;
        float l0 = 0.f, l1 = 0.f;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t x[32], y[16];
          tmem_ld32(x, s_at + 32 * c);
          tmem_wait_ld();
          if (masked) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (32 * c + i >= see) x[i] = 0xFF800000u;
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float p0 = exp2_approx(fmaf(__uint_as_float(x[2 * i]), sl2, -sub));
            const float p1 = exp2_approx(fmaf(__uint_as_float(x[2 * i + 1]), sl2, -sub));
            l0 += p0;
            l1 += p1;
            y[i] = W::pack(p0, p1);
          }
          tmem_st16(s_at + 16 * c, y);
        }
        l += l0 + l1;
        tmem_wait_st();
      }
      tc_fence_before();
      mbar_arrive(bar_p);
    }
    // the sums of the rows
    if (!mbar_wait(bar_o, (done - 1) & 1)) return false;
    tc_fence_after();
    if (active) {
      const bool whole = w.kv0 == 0 && w.kv1 == w.nkv;
      const bool none = !(l != 0.f);  // no key seen (a NaN sum is not that)
      const float inv = none ? 0.f : 1.f / l;
      const uint64_t at = (w.tok0 + t) * a.n_q_heads + w.h * a.G + g;
      const uint32_t slot = 2 * blockIdx.x + (w.kv0 == a.plan->start[blockIdx.x].kv && w.qt == a.plan->start[blockIdx.x].qt &&
                                              w.h == a.plan->start[blockIdx.x].h && w.r == a.plan->start[blockIdx.x].r ? 0 : 1);
      const uint64_t prow = (uint64_t)slot * kRows + half * 128 + tid;
#pragma unroll
      for (int c = 0; c < NSLAB * 2; ++c) {
        uint32_t x[32];
        tmem_ld32(x, o_at + 32 * c);
        tmem_wait_ld();
        if (valid && whole) {
          char* o = a.out + 2 * (at * D + 32 * c);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t y[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float lo = none ? 0.f : __uint_as_float(x[8 * i + 2 * k]) * inv;
              const float hi = none ? 0.f : __uint_as_float(x[8 * i + 2 * k + 1]) * inv;
              y[k] = W::pack(lo, hi);
            }
            if (32 * c + 8 * i < (int)D) *reinterpret_cast<uint4*>(o + 16 * i) = make_uint4(y[0], y[1], y[2], y[3]);
          }
        } else if (valid) {
          float* o = a.part + prow * D + 32 * c;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (32 * c + 4 * i < (int)D)
              *reinterpret_cast<uint4*>(o + 4 * i) = make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
        }
        __syncwarp();
      }
      if (valid) {
        const float top2 = top == -INFINITY ? -INFINITY : top * sl2 - W::kShift;
        if (whole) a.lse[at] = none ? -INFINITY : (top2 + log2_approx(l)) * kLn2;
        else a.part_ml[prow] = make_float2(none ? -INFINITY : top2, l);
      }
    }
    tc_fence_before();
  }
  return true;
}

template <typename T, int NSLAB>
__device__ __forceinline__ bool product_role(const AttnArgs& a, TileShared& sh, uint32_t q_smem, uint32_t ring) {
  using Sh = TileShape<NSLAB>;
  constexpr uint32_t kQk = mma_desc(Weights<T>::kBf16, 128, kKeys, false);
  constexpr uint32_t kPv = mma_desc(Weights<T>::kBf16, 128, NSLAB * 64, true);
  const uint32_t lane = threadIdx.x & 31, tmem = sh.tmem, steps = (a.kv.D + 15) / 16;
  uint32_t item = 0;                 // ring tiles taken so far
  uint32_t tiles[2] = {0, 0};        // query tiles of each half
  uint32_t keys[2] = {0, 0};         // key tiles of each half
  auto full = [&](uint32_t i) { return mbar_wait(smem_u32(&sh.full[i % Sh::kRing]), (i / Sh::kRing) & 1); };
  auto tile_at = [&](uint32_t i) { return ring + (i % Sh::kRing) * Sh::kTile; };
  auto scores = [&](uint32_t half, uint32_t k_item) {
    if (lane == 0) {
      for (uint32_t k = 0; k < steps; ++k) {
        const uint32_t off = (k / 4) * kSlabBytes + (k % 4) * 32;
        mma_ss(tmem + s_col(half), tile_desc(q_smem + half * Sh::kTile + off, 16), tile_desc(tile_at(k_item) + off, 16), kQk, k > 0);
      }
      mma_commit(smem_u32(&sh.s_full[half]));
    }
  };
  Walk w;
  for (bool more = w.begin(a); more; more = w.next(a)) {
    const uint32_t halves = w.rows - w.qt * kRows > 128 ? 2 : 1, L = w.kv1 - w.kv0;
    for (uint32_t s = 0; s < halves; ++s) {
      if (!mbar_wait(smem_u32(&sh.q_full[s]), tiles[s]++ & 1)) return false;
      if (s == 0 && !full(item)) return false;
      tc_fence_after();
      scores(s, item);
    }
    if (lane == 0) mma_commit(smem_u32(&sh.empty[item % Sh::kRing]));
    for (uint32_t j = 0; j < L; ++j, item += 2) {
      const uint32_t v_item = item + 1, k_next = item + 2;
      if (!full(v_item)) return false;
      const uint64_t first = (uint64_t)(w.kv0 + j) * kKeys;
      if (first + kKeys > w.n) {
        // slots that hold no token may hold NaN: zero their values (their weights are zero)
        const uint32_t have = w.n > first ? (uint32_t)(w.n - first) : 0;
        for (uint32_t i = have * (NSLAB * 8) + lane; i < kKeys * NSLAB * 8; i += 32) {
          const uint32_t row = i / (NSLAB * 8), c = i % (NSLAB * 8);
          const uint32_t at = tile_at(v_item) + (c / 8) * kSlabBytes + row * 128 + (c % 8) * 16;
          asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(at), "r"(0u) : "memory");
        }
        fence_async_shared();
        __syncwarp();
      }
      for (uint32_t s = 0; s < halves; ++s) {
        if (!mbar_wait(smem_u32(&sh.p_full[s]), keys[s]++ & 1)) return false;
        tc_fence_after();
        if (lane == 0) {
#pragma unroll
          for (uint32_t k = 0; k < kKeys / 16; ++k)
            mma_ts(tmem + o_col(s), tmem + s_col(s) + k * 8, tile_desc(tile_at(v_item) + k * 2048, kSlabBytes), kPv,
                   j > 0 || k > 0);
          mma_commit(smem_u32(&sh.pv_done[s]));
        }
        if (j + 1 < L) {
          if (s == 0 && !full(k_next)) return false;
          // in order after the product above, which reads the weights these scores overwrite
          scores(s, k_next);
        }
      }
      if (lane == 0) {
        mma_commit(smem_u32(&sh.empty[v_item % Sh::kRing]));
        if (j + 1 < L) mma_commit(smem_u32(&sh.empty[k_next % Sh::kRing]));
      }
    }
  }
  return true;
}

// Keys and values by tensor copies: a copy a stretch of `box` slots (a divisor
// of the page size and of the tile) and slab.  Stretches at or past the
// request's end and pages that the cache does not have read as zeros: their
// page coordinate is n_pages, which is out of range.
template <int NSLAB>
__device__ __forceinline__ bool copy_role(const AttnArgs& a, TileShared& sh, const CUtensorMap* mk, const CUtensorMap* mv,
                                          uint32_t ring, uint32_t& issued) {
  using Sh = TileShape<NSLAB>;
  const uint32_t lane = threadIdx.x & 31, boxes = kKeys / a.box;
  Walk w;
  for (bool more = w.begin(a); more; more = w.next(a)) {
    const uint32_t* ids = a.kv.page_ids + w.page0;
    for (uint32_t j = w.kv0; j < w.kv1; ++j) {
      const uint64_t key = (uint64_t)j * kKeys + lane * a.box;
      int page = (int)a.kv.n_pages, slot = 0;
      if (lane < boxes && key < w.n) {
        const uint32_t id = __ldg(ids + key / a.kv.B);
        if (id < a.kv.n_pages) page = (int)id;
        else report(a.status, PTC_ERR_INVALID_ARG);
        slot = (int)(key % a.kv.B);
      }
#pragma unroll
      for (int kv = 0; kv < 2; ++kv, ++issued) {
        const uint32_t at = issued % Sh::kRing;
        if (issued >= Sh::kRing && !mbar_wait(smem_u32(&sh.empty[at]), (issued / Sh::kRing - 1) & 1)) return false;
        const uint32_t bar = smem_u32(&sh.full[at]), dst = ring + at * Sh::kTile + lane * a.box * 128;
        if (lane == 0) mbar_expect(bar, Sh::kTile);
        __syncwarp();
        if (lane < boxes)
#pragma unroll
          for (int s = 0; s < NSLAB; ++s)
            tma_load_4d(dst + s * kSlabBytes, kv == 0 ? mk : mv, bar, 64 * s, slot, (int)w.h, page);
      }
    }
  }
  return true;
}

// The same for page sizes that are no multiple of 8 (a swizzled tile takes
// copies of whole groups of 8 rows): 96 threads copy 16 bytes each.
template <int NSLAB>
__device__ __forceinline__ bool gather_role(const AttnArgs& a, TileShared& sh, uint32_t ring) {
  using Sh = TileShape<NSLAB>;
  const uint32_t tid = threadIdx.x - 288;
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
        if (issued >= Sh::kRing && !mbar_wait(smem_u32(&sh.empty[at]), (issued / Sh::kRing - 1) & 1)) return false;
        const char* src = kv == 0 ? a.kv.k : a.kv.v;
        const int64_t sp = kv == 0 ? a.kv.ks_page : a.kv.vs_page, ss = kv == 0 ? a.kv.ks_slot : a.kv.vs_slot;
        const int64_t head = w.h * (kv == 0 ? a.kv.ks_head : a.kv.vs_head);
        for (uint32_t i = tid; i < kKeys * NSLAB * 8; i += 96) {
          const uint32_t row = i / (NSLAB * 8), c = i % (NSLAB * 8);
          const uint64_t key = (uint64_t)j * kKeys + row;
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

template <typename T, int NSLAB, bool TMA>
__global__ void __launch_bounds__(kTileThreads, 1) k_attn_tiles(const __grid_constant__ CUtensorMap mk,
                                                                const __grid_constant__ CUtensorMap mv, AttnArgs a) {
  using Sh = TileShape<NSLAB>;
  extern __shared__ char smem_raw[];
  __shared__ TileShared sh;
  const uint32_t q_smem = (smem_u32(smem_raw) + 1023) & ~1023u, ring = q_smem + 2 * Sh::kTile;
  const uint32_t warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < Sh::kRing; ++i) {
      mbar_init(smem_u32(&sh.full[i]), TMA ? 1 : 96);
      mbar_init(smem_u32(&sh.empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sh.q_full[i]), 128);
      mbar_init(smem_u32(&sh.s_full[i]), 1);
      mbar_init(smem_u32(&sh.p_full[i]), 128);
      mbar_init(smem_u32(&sh.pv_done[i]), 1);
    }
    mbar_init(smem_u32(&sh.drain), 1);
    sh.abort = 0;
    fence_mbar_init();
  }
  if (warp == 8) tmem_alloc(smem_u32(&sh.tmem), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  grid_dep_sync();
  const bool go = a.plan->ok != 0;
  uint32_t issued = 0;
  if (go) {
    bool fine = true;
    if (warp < 8) {
      fine = softmax_role<T, NSLAB>(a, sh, q_smem, warp / 4);
    } else if (warp == 8) {
      fine = product_role<T, NSLAB>(a, sh, q_smem, ring);
      // every product and every arrival it owes is done before the CTA ends
      if ((threadIdx.x & 31) == 0) mma_commit(smem_u32(&sh.drain));
      __syncwarp();
      fine &= mbar_wait(smem_u32(&sh.drain), 0);
    } else if (TMA) {
      if (warp == 9) fine = copy_role<NSLAB>(a, sh, &mk, &mv, ring, issued);
    } else {
      fine = gather_role<NSLAB>(a, sh, ring);
    }
    if (!fine) {
      sh.abort = 1;
      report(a.status, PTC_ERR_TIMEOUT);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (sh.abort && TMA && warp == 9) {
    // given up: let the copies in flight land
    for (uint32_t i = issued > Sh::kRing ? issued - Sh::kRing : 0; i < issued; ++i)
      (void)mbar_wait(smem_u32(&sh.full[i % Sh::kRing]), (i / Sh::kRing) & 1);
  }
  if (sh.abort && !TMA) cp_async_wait<0>();
  __syncthreads();
  if (warp == 8) tmem_free(sh.tmem, 512);
}

// The rows of split tiles: CTA c looks whether its start is the first cut of
// a tile, and then puts that tile's parts together.  blockIdx.y: 32 rows.
template <typename T>
__global__ void __launch_bounds__(256) k_attn_join(AttnArgs a) {
  grid_dep_sync();
  if (!a.plan->ok) return;
  const uint32_t c = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = a.kv.D;
  const uint64_t U = a.plan->units, C = a.ctas;
  const CtaStart s = a.plan->start[c];
  if (s.u == U * (c + 1) / C || s.kv == 0) return;
  auto cta_of = [&](uint64_t u) { return (uint32_t)(((u + 1) * C - 1) / U); };
  const uint64_t first = s.u - s.kv;
  const uint32_t c0 = cta_of(first);
  if (cta_of(s.u - 1) != c0) return;
  const uint64_t tok0 = a.tok_off[s.r];
  const uint32_t m = (uint32_t)(a.tok_off[s.r + 1] - tok0), n = a.kv.kv_len[s.r], rows = m * a.G;
  const uint32_t nkv = key_tiles(m, n, a.G, s.qt), c1 = cta_of(first + nkv - 1);
  for (uint32_t i = blockIdx.y * 32 + warp; i < blockIdx.y * 32 + 32; i += 8) {
    const uint32_t row = s.qt * kRows + i;
    if (row >= rows) break;
    auto slot_row = [&](uint32_t x) {
      return (uint64_t)(2 * x + (x == c0 && a.plan->start[x].u != first ? 1 : 0)) * kRows + i;
    };
    auto empty = [&](uint32_t x) { return U * x / C == U * (x + 1) / C; };
    float top = -INFINITY;
    for (uint32_t x = c0; x <= c1; ++x)
      if (!empty(x)) top = fmaxf(top, a.part_ml[slot_row(x)].x);
    float l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (uint32_t x = c0; x <= c1; ++x) {
      if (empty(x)) continue;
      const uint64_t at = slot_row(x);
      const float2 ml = a.part_ml[at];
      if (ml.x == -INFINITY) continue;  // its part of the row saw no key
      const float f = exp2_approx(ml.x - top);
      l = fmaf(ml.y, f, l);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (lane + 32 * k < D) o[k] = fmaf(a.part[at * D + lane + 32 * k], f, o[k]);
    }
    const bool none = top == -INFINITY;
    const float inv = none ? 0.f : 1.f / l;
    const uint64_t at = (tok0 + row / a.G) * a.n_q_heads + s.h * a.G + row % a.G;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (lane + 32 * k < D) reinterpret_cast<T*>(a.out)[at * D + lane + 32 * k] = static_cast<T>(o[k] * inv);
    if (lane == 0) a.lse[at] = none ? -INFINITY : (top + log2_approx(l)) * kLn2;
  }
}

template <typename T>
__device__ __forceinline__ float to_f(T x) { return static_cast<float>(x); }

template <typename T>
__device__ __forceinline__ float dot8(const uint4& a, const uint4& b, float acc) {
  const T* x = reinterpret_cast<const T*>(&a);
  const T* y = reinterpret_cast<const T*>(&b);
#pragma unroll
  for (int i = 0; i < 8; ++i) acc = fmaf(to_f(x[i]), to_f(y[i]), acc);
  return acc;
}

// One thread a slot and key head: its weights over every row that sees it.
template <typename T>
__global__ void __launch_bounds__(128) k_attn_mass(AttnArgs a) {
  grid_dep_sync();
  if (!a.plan->ok) return;
  const uint32_t h = blockIdx.y;
  const uint64_t total = a.kv.page_off[a.kv.n_req] - a.kv.page_off[0];
  const uint64_t slot = (uint64_t)blockIdx.x * 128 + threadIdx.x;
  if (slot >= total * a.kv.B) return;
  const uint64_t page_at = a.kv.page_off[0] + slot / a.kv.B;
  const uint32_t r = req_search(a.kv.page_off, 0, a.kv.n_req - 1, page_at);
  const int64_t j = (int64_t)((page_at - a.kv.page_off[r]) * a.kv.B + slot % a.kv.B);
  const uint64_t at = h * a.mass_stride + page_at * a.kv.B + slot % a.kv.B;
  const int64_t n = a.kv.kv_len[r], t0 = a.tok_off[r], m = (int64_t)a.tok_off[r + 1] - t0;
  float sum = 0.f;
  if (j < n) {
    const uint32_t page = a.kv.page_ids[page_at];
    if (page < a.kv.n_pages) {
      const char* k = a.kv.k + 2 * (page * a.kv.ks_page + h * a.kv.ks_head + (j % a.kv.B) * a.kv.ks_slot);
      for (int64_t i = j > n - m ? j - (n - m) : 0; i < m; ++i)
        for (uint32_t g = 0; g < a.G; ++g) {
          const char* q = a.q + 2 * ((t0 + i) * a.q_tok + (h * a.G + g) * a.q_head);
          float s = 0.f;
          for (uint32_t d = 0; d < a.kv.D; d += 8)
            s = dot8<T>(*reinterpret_cast<const uint4*>(q + 2 * d), *reinterpret_cast<const uint4*>(k + 2 * d), s);
          sum += expf(s * a.scale - a.lse[(t0 + i) * a.n_q_heads + h * a.G + g]);
        }
    }
    if (a.mass_in) sum += a.mass_in[at];
  }
  a.mass_out[at] = sum;
}

// cuTensorMapEncodeTiled, from the driver that the runtime has loaded.
using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeFn encoder() {
  static const EncodeFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &r) != cudaSuccess ||
        r != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      return static_cast<EncodeFn>(nullptr);
    }
    return reinterpret_cast<EncodeFn>(p);
  }();
  return fn;
}

// The cache as [page][head][slot][d], read 64 columns by `box` slots at a time.
bool cache_map(CUtensorMap* map, const KvView& kv, bool bf16, char* base, int64_t page, int64_t head, int64_t slot,
               uint32_t box) {
  const cuuint64_t dims[4] = {kv.D, kv.B, kv.H, kv.n_pages};
  const cuuint64_t strides[3] = {2 * (cuuint64_t)slot, 2 * (cuuint64_t)head, 2 * (cuuint64_t)page};
  const cuuint32_t boxes[4] = {64, box, 1, 1}, steps[4] = {1, 1, 1, 1};
  const EncodeFn fn = encoder();
  return fn && fn(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, base, dims, strides,
                  boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int NSLAB, bool TMA>
ptc_status launch_tiles(const AttnArgs& a, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t s) {
  if (cudaFuncSetAttribute(k_attn_tiles<T, NSLAB, TMA>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           TileShape<NSLAB>::kSmem) != cudaSuccess)
    return PTC_ERR_CUDA;
  PTC_KERNEL("k_attn_tiles", s, (k_attn_tiles<T, NSLAB, TMA>), a.ctas, kTileThreads, TileShape<NSLAB>::kSmem, mk, mv, a);
  return PTC_OK;
}

template <typename T>
ptc_status launch(AttnArgs& a, cudaStream_t s) {
  PTC_KERNEL("k_attn_plan", s, k_attn_plan, 1, kPlanThreads, 0, a);
  if (a.n_tok) {
    CUtensorMap mk{}, mv{};
    // copies of whole groups of 8 rows that neither leave a page nor a tile
    a.box = 128;
    while (a.kv.B % a.box) a.box /= 2;
    const bool tma = a.box >= 8 && a.kv.n_pages > 0;
    if (tma && (!cache_map(&mk, a.kv, Weights<T>::kBf16, a.kv.k, a.kv.ks_page, a.kv.ks_head, a.kv.ks_slot, a.box) ||
                !cache_map(&mv, a.kv, Weights<T>::kBf16, a.kv.v, a.kv.vs_page, a.kv.vs_head, a.kv.vs_slot, a.box)))
      return PTC_ERR_CUDA;
    const ptc_status st = a.kv.D > 64 ? (tma ? launch_tiles<T, 2, true>(a, mk, mv, s) : launch_tiles<T, 2, false>(a, mk, mv, s))
                                      : (tma ? launch_tiles<T, 1, true>(a, mk, mv, s) : launch_tiles<T, 1, false>(a, mk, mv, s));
    if (st != PTC_OK) return st;
    PTC_KERNEL("k_attn_join", s, k_attn_join<T>, dim3(a.ctas, kRows / 32), 256, 0, a);
  }
  if (a.mass_out && a.kv.n_page_ids)
    PTC_KERNEL("k_attn_mass", s, k_attn_mass<T>, dim3((uint32_t)((a.kv.n_page_ids * a.kv.B + 127) / 128), a.kv.H), 128,
               0, a);
  return PTC_OK;
}

// Workspace: the status word, the plan, the unit offsets and the parts.
struct AttnWs {
  size_t plan, units, ml, part, total;
};
AttnWs attn_ws(uint32_t n_req, uint32_t ctas, uint32_t D) {
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  AttnWs w;
  w.plan = kKvStatusBytes;
  w.units = w.plan + up(sizeof(AttnPlan));
  w.ml = w.units + up((size_t)(n_req + 1) * 8);
  w.part = w.ml + up((size_t)2 * ctas * kRows * 8);
  w.total = w.part + up((size_t)2 * ctas * kRows * D * 4);
  return w;
}
uint32_t tile_ctas() {
  const int n = num_sms();
  return n < (int)kMaxCtas ? (uint32_t)n : kMaxCtas;
}

}  // namespace
}  // namespace ptc

using namespace ptc;

extern "C" size_t ptc_paged_attention_workspace_bytes(uint32_t n_req, uint64_t, uint32_t, uint32_t, uint32_t head_dim) {
  return attn_ws(n_req, tile_ctas(), head_dim).total;
}

extern "C" ptc_status ptc_paged_attention(const ptc_paged_kv* kv, const void* q, const int64_t q_stride[2],
                                          const uint64_t* tok_off, uint64_t n_tok, uint32_t n_q_heads,
                                          uint32_t max_q_len, float scale, void* out, float* lse,
                                          const float* mass_in, float* mass_out, uint64_t mass_stride, void* ws,
                                          size_t ws_bytes, uint32_t* status, void* stream) {
  AttnArgs a{};
  const ptc_status st = kv_view(kv, &a.kv);
  if (st != PTC_OK) return st;
  if (!tok_off || !q_stride || n_q_heads < 1 || n_q_heads % kv->n_kv_heads) return PTC_ERR_INVALID_ARG;
  if (!(scale > 0.f) || !std::isfinite(scale) || (n_tok && !kv->n_req)) return PTC_ERR_INVALID_ARG;
  if (n_tok > (uint64_t(1) << 31) || n_tok * n_q_heads > (uint64_t(1) << 31) || kv->n_page_ids * kv->block_size > (uint64_t(1) << 38))
    return PTC_ERR_OVERFLOW;
  if (mass_out ? mass_stride / kv->block_size < kv->n_page_ids : mass_in != nullptr) return PTC_ERR_INVALID_ARG;
  if (kv->n_pages > 0x7FFFFFFFu) return PTC_ERR_OVERFLOW;  // tensor copies have signed coordinates
  const AttnWs at = attn_ws(kv->n_req, tile_ctas(), kv->head_dim);
  if (!ws_ok(ws, ws_bytes, at.total)) return PTC_ERR_WORKSPACE;
  if (kv->n_req == 0) return PTC_OK;
  if (n_tok && (!aligned16(q) || !aligned16(out) || !lse)) return PTC_ERR_INVALID_ARG;
  const uint32_t ext[2] = {(uint32_t)n_tok, n_q_heads};
  for (int i = 0; i < 2; ++i)
    if (!stride_ok(q_stride[i], ext[i])) return PTC_ERR_INVALID_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  a.q = static_cast<const char*>(q);
  a.q_tok = stride_of(q_stride[0], ext[0]);
  a.q_head = stride_of(q_stride[1], ext[1]);
  a.tok_off = tok_off;
  a.n_tok = n_tok;
  a.n_q_heads = n_q_heads;
  a.G = n_q_heads / kv->n_kv_heads;
  a.max_q_len = max_q_len;
  a.scale = scale;
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.mass_in = mass_in;
  a.mass_out = mass_out;
  a.mass_stride = mass_stride;
  char* w = static_cast<char*>(ws);
  a.ctas = tile_ctas();
  a.plan = reinterpret_cast<AttnPlan*>(w + at.plan);
  a.unit_off = reinterpret_cast<uint64_t*>(w + at.units);
  a.part_ml = reinterpret_cast<float2*>(w + at.ml);
  a.part = reinterpret_cast<float*>(w + at.part);
  if (kv_begin(status, ws, s, &a.status) != PTC_OK) return PTC_ERR_CUDA;
  const ptc_status run = kv->dtype == PTC_DTYPE_BF16 ? launch<__nv_bfloat16>(a, s) : launch<__half>(a, s);
  if (run != PTC_OK) return run;
  return kv_end(status, a.status, s);
}
