// Accumulated attention weights (ptc_paged_attention with mass_out): for every
// cached token and key head the sum of its weights over the call's queries,
//   sum over rows i of exp2(scale log2(e) s_ij - log2(e) lse_i),
// once the rows' lse are known.  Two ways:
//   few rows    requests of up to kFewRows rows (single tokens): the tile
//               kernel leaves the scores, 4 bytes a row, token and key head,
//               and one pass adds them up.  Reading the keys again would be 2 D
//               bytes a token and key head: 256 at D = 128, against 8 a row
//               written and read.  32 single tokens over 202K: 139 us without
//               the weights, 161 with them.
//   many rows   the scores are computed again, transposed: one thread a token
//               adds up its column of rows without a word to its neighbours.
#include <cstddef>
#include <type_traits>

#include "ptc_attn.cuh"

namespace ptc {
namespace {

// A slot of no request.
__device__ __forceinline__ void copy_weight(const AttnArgs& a, uint64_t at) {
  if (a.mass_in != a.mass_out) a.mass_out[at] = a.mass_in ? a.mass_in[at] : 0.f;
}

// ------------------------------------------------------------------ few rows
constexpr int kRowThreads = 256;
constexpr uint32_t kRowSlots = 4 * kRowThreads;

__global__ void __launch_bounds__(kRowThreads) k_mass_rows(const AttnArgs a) {
  grid_dep_sync();
  if (!a.plan->ok) return;
  __shared__ uint32_t s_r;
  const uint32_t R = a.kv.n_req, B = a.kv.B, h = blockIdx.y;
  const uint64_t first = a.kv.page_off[0] * B, end = a.kv.page_off[R] * B;
  const uint64_t s0 = (uint64_t)blockIdx.x * kRowSlots, slots = a.kv.n_page_ids * B;
  if ((s0 + kRowSlots <= first || s0 >= end) && a.mass_in == a.mass_out) return;  // no request's, and in place
  if (threadIdx.x == 0) s_r = req_search(a.kv.page_off, 0, R - 1, s0 / B);
  __syncthreads();
  uint32_t r = s_r;
  const bool four = B % 4 == 0 && a.mass_stride % 4 == 0 && (((uintptr_t)a.mass_in | (uintptr_t)a.mass_out) & 15) == 0;
  const uint32_t width = four ? 4 : 1;
  for (uint32_t pass = 0; pass < 4 / width; ++pass) {
    const uint64_t slot = s0 + ((uint64_t)pass * kRowThreads + threadIdx.x) * width;
    if (slot >= slots) return;
    if (slot < first || slot >= end) {
      for (uint32_t k = 0; k < width; ++k) copy_weight(a, h * a.mass_stride + slot + k);
      continue;
    }
    while (r + 1 < R && a.kv.page_off[r + 1] * B <= slot) ++r;
    const int64_t j = (int64_t)(slot - a.kv.page_off[r] * B), n = a.kv.kv_len[r];
    const uint64_t tok0 = a.tok_off[r];
    const int64_t m = (int64_t)(a.tok_off[r + 1] - tok0);
    const uint64_t at = h * a.mass_stride + slot;
    const float* score = a.scores + (uint64_t)h * a.few * a.mass_stride + slot;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    if (j < n) {
      const float sl2 = a.scale * kLog2e;
      const int64_t sees0 = n - m + 1;  // keys that the first token sees
      const uint32_t rows = (uint32_t)m * a.G;
      const float* lse = a.lse + tok0 * a.n_q_heads + h * a.G;
      for (uint32_t i0 = 0; i0 < rows; i0 += 4) {
        float4 x[4];
        float off[4];
        int64_t sees[4];
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {  // four rows' loads in flight
          const uint32_t i = i0 + u < rows ? i0 + u : i0, t = i / a.G;
          sees[u] = i0 + u < rows ? sees0 + t : 0;
          off[u] = lse[(uint64_t)t * a.n_q_heads + (i - t * a.G)] * kLog2e;
          const float* p = score + i * a.mass_stride;
          // what lies past the row's last key is not used
          x[u] = four ? *reinterpret_cast<const float4*>(p) : make_float4(*p, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
          const float y[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if ((uint32_t)k < width && j + k < sees[u]) sum[k] += exp2_approx(fmaf(y[k], sl2, -off[u]));
        }
      }
    }
    if (four) {
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      if (j < n && a.mass_in) o = *reinterpret_cast<const float4*>(a.mass_in + at);
      o.x = j < n ? o.x + sum[0] : 0.f;
      o.y = j + 1 < n ? o.y + sum[1] : 0.f;
      o.z = j + 2 < n ? o.z + sum[2] : 0.f;
      o.w = j + 3 < n ? o.w + sum[3] : 0.f;
      *reinterpret_cast<float4*>(a.mass_out + at) = o;
    } else {
      a.mass_out[at] = j < n ? (a.mass_in ? a.mass_in[at] : 0.f) + sum[0] : 0.f;
    }
  }
}

// ------------------------------------------------------------------ many rows
// One CTA an SM walks its units, pairs of 256 keys and half a query tile.
// Scores transposed, S = K Q^T: 128 keys in the lanes of tensor memory, up to
// 128 query rows in its columns, for both halves of the keys and two units at a
// time.  Four groups of 4 warps, one a half of the rows and every other unit,
// add up exp2(s - lse) along rows of S, which are columns of the scores; a thread
// has a key of either half, so that an lse is read once for two scores.  Warp 16
// issues the products, warp 17 loads keys (with warp 19 where there are no
// tensor copies), warp 18 queries.
// What bounds it is shared memory, 128 bytes a cycle: a unit's products read 128
// KB, its queries are 32 KB, the lse 32 KB (at D = 128), 1,540 cycles for 1,024
// of products and as many of exponentials.  (With 128 keys a unit the queries'
// stream out of L2, 7.4 TB/s, was the bound.)  A unit takes 2,270 cycles: 4
// chunks of 300 to 2,048 tokens over up to 8K, 212 us beside 296 for the
// attention itself.
constexpr int kMassThreads = 640;
constexpr int kSlab = 128 * 128;
constexpr uint32_t kQueryRing = 3;

struct MassShared {
  uint64_t k_full[2], k_empty[2], q_full[kQueryRing], q_empty[kQueryRing], s_full[4], s_empty[4], drain;
  alignas(16) float lse[2][128];  // negated, in powers of two: of even and odd units (read four at a time)
  float sum[2][128];  // of one group: both halves of the keys
  uint32_t tmem;
};

template <int NSLAB>
struct MassShape {
  static constexpr int kTile = NSLAB * kSlab;
  static constexpr int kQueries = 4 * kTile;  // behind two key tiles of two halves
  static constexpr int kRest = kQueries + kQueryRing * kTile;
  static constexpr int kSmem = kRest + sizeof(MassShared);
  static_assert(kSmem <= 227 * 1024, "shared memory of a block");
  static_assert(kRest % 16 == 0 && offsetof(MassShared, lse) % 16 == 0, "16-byte reads");
};

struct MassWalk {
  uint64_t left, tok0, page0;
  uint32_t r, h, kt, q0, q1;  // half query tiles [q0, q1)
  uint32_t first, count;      // the first one that sees the key tile, and how many do
  uint32_t extra;             // units before the first of them
  uint32_t m, n;
  __device__ __forceinline__ void request(const AttnArgs& a) {
    tok0 = a.tok_off[r];
    m = (uint32_t)(a.tok_off[r + 1] - tok0);
    n = a.kv.kv_len[r];
    page0 = a.kv.page_off[r];
  }
  __device__ __forceinline__ void part(const AttnArgs& a, uint32_t minor) {
    first = first_seeing(m, n, a.tq, kt);
    count = div_up(m, a.tq) - first;
    q0 = first + minor;
    extra = minor ? 0 : kMassExtra;
    q1 = count - minor + extra > left ? q0 + (uint32_t)left - extra : first + count;
  }
  __device__ __forceinline__ bool begin(const AttnArgs& a) {
    const AttnPlan* p = a.plan + 1;
    const CtaStart s = p->start[blockIdx.x];
    left = p->start[blockIdx.x + 1].u - s.u;
    if (left == 0) return false;
    r = s.r;
    h = s.h;
    kt = s.major;
    tok0 = s.tok0;
    m = s.m;
    n = s.n;
    page0 = s.page0;
    part(a, s.minor);
    return true;
  }
  __device__ __forceinline__ bool next(const AttnArgs& a) {
    left -= q1 - q0 + extra;
    if (left == 0) return false;
    if ((uint64_t)++kt * kMassKeys >= n) {
      kt = 0;
      if (++h == a.kv.H) {
        h = 0;
        do {
          if (++r == a.kv.n_req) return false;
          request(a);
        } while (m == 0 || n == 0);
      }
    }
    part(a, 0);
    return true;
  }
  // Whether there are keys in the tile's second half.
  __device__ __forceinline__ bool two() const { return n > kt * kMassKeys + kKeys; }
  __device__ __forceinline__ uint32_t rows(const AttnArgs& a, uint32_t q) const {
    const uint32_t t = m - q * a.tq;
    return (t < a.tq ? t : a.tq) * a.G;
  }
};

// The weights of 32 rows added to the sums of a key of either half.
__device__ __forceinline__ void add_weights(const uint32_t (&x)[2][32], const float* lse, float sl2, float2 (&sum)[2][2]) {
  const float4* off = reinterpret_cast<const float4*>(lse);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const float4 o = off[k];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const float2 e0 = fma2(make_float2(__uint_as_float(x[half][4 * k]), __uint_as_float(x[half][4 * k + 1])),
                             make_float2(sl2, sl2), make_float2(o.x, o.y));
      const float2 e1 = fma2(make_float2(__uint_as_float(x[half][4 * k + 2]), __uint_as_float(x[half][4 * k + 3])),
                             make_float2(sl2, sl2), make_float2(o.z, o.w));
      sum[half][0] = add2(sum[half][0], make_float2(exp2_approx(e0.x), exp2_approx(e0.y)));
      sum[half][1] = add2(sum[half][1], make_float2(exp2_approx(e1.x), exp2_approx(e1.y)));
    }
  }
}

__device__ __forceinline__ bool mass_sums(const AttnArgs& a, MassShared& sh, uint32_t group) {
  const uint32_t tid = threadIdx.x & 127, side = group & 1, odd = group >> 1;
  const uint32_t tmem = sh.tmem + ((tid & ~31u) << 16) + odd * 256;
  const float sl2 = a.scale * kLog2e;
  auto odd_sync = [&] { asm volatile("bar.sync %0, 256;" ::"r"(2 + odd) : "memory"); };
  auto all_sync = [] { asm volatile("bar.sync 1, 512;" ::: "memory"); };
  uint32_t unit = 0, seg = 0, uses[2] = {0, 0};
  bool alive = true;  // a warp that has given up waiting runs on without, for the others at the barriers
  MassWalk w;
  for (bool more = w.begin(a); more; more = w.next(a), ++seg) {
    const uint32_t key = w.kt * kMassKeys + tid;  // and key + kKeys
    const int64_t t_first = (int64_t)key - ((int64_t)w.n - w.m);  // the first token that sees the key
    const bool two = w.two();
    // lse of a query tile's row `tid`; rows that are none count nothing below
    auto lse_of = [&](uint32_t q) {
      if (tid >= w.rows(a, q)) return 0.f;
      const uint64_t t = w.tok0 + (uint64_t)q * a.tq + tid / a.G;
      return -kLog2e * a.lse[t * a.n_q_heads + w.h * a.G + tid % a.G];
    };
    uint32_t q = w.q0 + ((odd ^ unit) & 1);
    float ahead = side == 0 && q < w.q1 ? lse_of(q) : 0.f;
    float2 sum[2][2] = {};
    for (; q < w.q1; q += 2) {
      if (side == 0) sh.lse[odd][tid] = ahead;
      odd_sync();
      if (side == 0 && q + 2 < w.q1) ahead = lse_of(q + 2);
      if (alive) alive = mbar_wait(smem_u32(&sh.s_full[2 * odd]), uses[0]++ & 1, a.limit);
      if (two && alive) alive = mbar_wait(smem_u32(&sh.s_full[2 * odd + 1]), uses[1]++ & 1, a.limit);
      tc_fence_after();
      // the rows that see either key, from `lo` on
      const int64_t lo64 = (t_first - (int64_t)q * a.tq) * a.G, lo64b = lo64 + (int64_t)kKeys * a.G;
      const int lo = lo64 <= 0 ? 0 : lo64 >= 128 ? 128 : (int)lo64, lo_b = lo64b <= 0 ? 0 : lo64b >= 128 ? 128 : (int)lo64b;
      const int rows = (int)w.rows(a, q), from = 64 * (int)side, to = rows < from + 64 ? rows : from + 64;
      const bool masked = __any_sync(kFull, lo > from || (two && lo_b > from) || ((rows & 31) && to == rows));
#pragma unroll 1
      for (int c = from; c < to; c += 32) {
        uint32_t x[2][32];
        tmem_ld32(x[0], tmem + c);
        tmem_ld32(x[1], tmem + 128 + c);  // (where there is no second half, anything, and not used)
        tmem_wait_ld(x[0]);
        tmem_wait_ld(x[1]);
        if (!masked) {
          add_weights(x, sh.lse[odd] + c, sl2, sum);
        } else {
#pragma unroll
          for (int k = 0; k < 32; ++k) {
            const float off = sh.lse[odd][c + k];
            const float p0 = exp2_approx(fmaf(__uint_as_float(x[0][k]), sl2, off));
            const float p1 = exp2_approx(fmaf(__uint_as_float(x[1][k]), sl2, off));
            if (c + k >= lo && c + k < rows) sum[0][0].x += p0;
            if (c + k >= lo_b && c + k < rows) sum[1][0].x += p1;
          }
        }
      }
      tc_fence_before();
      mbar_arrive_warp(smem_u32(&sh.s_empty[2 * odd]));
      if (two) mbar_arrive_warp(smem_u32(&sh.s_empty[2 * odd + 1]));
      odd_sync();  // the lse have been read
    }
    unit += w.q1 - w.q0;
    // the four groups' sums (where there is no second half, its are not used)
    float total[2];
#pragma unroll
    for (int half = 0; half < 2; ++half)
      total[half] = (sum[half][0].x + sum[half][0].y) + (sum[half][1].x + sum[half][1].y);
    all_sync();
    float (*place)[128] = side == 0 ? sh.lse : sh.sum;
    if (odd) place[0][tid] = total[0], place[1][tid] = total[1];
    all_sync();
    if (!odd) total[0] += place[0][tid], total[1] += place[1][tid];
    all_sync();
    if (group == 1) place[0][tid] = total[0], place[1][tid] = total[1];
    all_sync();
    if (group == 0) {
      const bool whole = w.q0 == w.first && w.q1 == w.first + w.count;
#pragma unroll
      for (uint32_t half = 0; half < 2; ++half) {
        const uint32_t k = key + half * kKeys;
        total[half] += sh.sum[half][tid];
        if (!whole) {
          a.part_mass[(2 * (uint64_t)blockIdx.x + (seg == 0 ? 0 : 1)) * kMassKeys + half * kKeys + tid] = total[half];
        } else if (k < w.n) {
          const uint64_t at = w.h * a.mass_stride + w.page0 * a.kv.B + k;
          a.mass_out[at] = (a.mass_in ? a.mass_in[at] : 0.f) + total[half];
        }
      }
    }
    all_sync();
  }
  return alive;
}

template <typename T, int NSLAB>
__device__ __forceinline__ bool mass_products(const AttnArgs& a, MassShared& sh, uint32_t smem) {
  using Sh = MassShape<NSLAB>;
  constexpr bool bf16 = !std::is_same<T, __half>::value;
  const uint32_t tmem = sh.tmem, steps = (a.kv.D + 15) / 16;
  uint32_t unit = 0, seg = 0, used[4] = {0, 0, 0, 0};
  MassWalk w;
  for (bool more = w.begin(a); more; more = w.next(a), ++seg) {
    const uint32_t k_at = smem + (seg & 1) * 2 * Sh::kTile, halves = w.two() ? 2 : 1;
    if (!mbar_wait(smem_u32(&sh.k_full[seg & 1]), (seg >> 1) & 1, a.limit)) return false;
    for (uint32_t q = w.q0; q < w.q1; ++q, ++unit) {
      const uint32_t ring = unit % kQueryRing, q_at = smem + Sh::kQueries + ring * Sh::kTile;
      if (!mbar_wait(smem_u32(&sh.q_full[ring]), (unit / kQueryRing) & 1, a.limit)) return false;
      const uint32_t desc = mma_desc(bf16, 128, (w.rows(a, q) + 15) & ~15u, false);
      const uint64_t db = tile_desc(q_at, 16);
#pragma unroll
      for (uint32_t half = 0; half < 2; ++half) {
        if (half >= halves) break;
        const uint32_t buf = (unit & 1) * 2 + half;
        uint32_t& n = (unit & 1) ? used[2 + half] : used[half];
        if (n && !mbar_wait(smem_u32(&sh.s_empty[buf]), (n - 1) & 1, a.limit)) return false;
        ++n;
        tc_fence_after();
        const uint64_t da = tile_desc(k_at + half * Sh::kTile, 16);
        if (elect_lane()) {
          mma_ss<false>(tmem + buf * 128, da, db, desc);
#pragma unroll
          for (uint32_t k = 1; k < NSLAB * 4; ++k) {
            const uint32_t off = (k / 4) * kSlab + (k % 4) * 32;
            if (k < steps) mma_ss<true>(tmem + buf * 128, desc_at(da, off), desc_at(db, off), desc);
          }
          mma_commit(smem_u32(&sh.s_full[buf]));
          if (half + 1 == halves) {
            mma_commit(smem_u32(&sh.q_empty[ring]));
            if (q + 1 == w.q1) mma_commit(smem_u32(&sh.k_empty[seg & 1]));
          }
        }
        __syncwarp();
      }
    }
  }
  return true;
}

template <int NSLAB>
__device__ __forceinline__ bool mass_queries(const AttnArgs& a, MassShared& sh, const CUtensorMap* mq, uint32_t smem,
                                             uint32_t& unit) {
  using Sh = MassShape<NSLAB>;
  const uint32_t lane = threadIdx.x & 31;
  if (a.withhold) return true;
  MassWalk w;
  for (bool more = w.begin(a); more; more = w.next(a))
    for (uint32_t q = w.q0; q < w.q1; ++q, ++unit) {
      const uint32_t at = unit % kQueryRing, bar = smem_u32(&sh.q_full[at]), dst = smem + Sh::kQueries + at * Sh::kTile;
      if (unit >= kQueryRing && !mbar_wait(smem_u32(&sh.q_empty[at]), (unit / kQueryRing - 1) & 1, a.limit)) return false;
      if (lane == 0) {
        mbar_expect(bar, NSLAB * a.tq * a.G * 128);
#pragma unroll
        for (int c = 0; c < NSLAB; ++c)
          tma_load_4d(dst + c * kSlab, mq, bar, 64 * c, 0, (int)w.h, (int)(w.tok0 + (uint64_t)q * a.tq));
      }
      __syncwarp();
    }
  return true;
}

// Key tiles, by tensor copies (one warp) or 16 bytes at a time (two, each tile
// waited for: pages of 12 take the call of 4 chunks above from 508 us to 2.5 ms).
// Pages that the cache does not have were reported by the tile kernel.
template <int NSLAB, bool TMA>
__device__ __forceinline__ bool mass_keys(const AttnArgs& a, MassShared& sh, const CUtensorMap* mk, uint32_t smem,
                                          uint32_t& seg) {
  using Sh = MassShape<NSLAB>;
  const uint32_t lane = threadIdx.x & 31;
  const uint32_t tid = lane + (threadIdx.x >= 608 ? 32 : 0);
  MassWalk w;
  for (bool more = w.begin(a); more; more = w.next(a), ++seg) {
    const uint32_t at = seg & 1, bar = smem_u32(&sh.k_full[at]), halves = w.two() ? 2 : 1;
    const uint32_t* ids = a.kv.page_ids + w.page0;
    if (seg >= 2 && !mbar_wait(smem_u32(&sh.k_empty[at]), ((seg >> 1) - 1) & 1, a.limit)) return false;
    if constexpr (TMA) {
      const uint32_t boxes = kKeys / a.box;
      if (lane == 0) mbar_expect(bar, halves * Sh::kTile);
      __syncwarp();
      for (uint32_t half = 0; half < halves; ++half) {
        const uint32_t dst = smem + (at * 2 + half) * Sh::kTile;
        const uint32_t key = w.kt * kMassKeys + half * kKeys + lane * a.box;
        int page = (int)a.kv.n_pages, slot = 0;
        if (lane < boxes && key < w.n) {
          const uint32_t id = __ldg(ids + key / a.kv.B);
          if (id < a.kv.n_pages) page = (int)id;
          slot = (int)(key % a.kv.B);
        }
        if (lane < boxes)
#pragma unroll
          for (int s = 0; s < NSLAB; ++s)
            tma_load_4d(dst + s * kSlab + lane * a.box * 128, mk, bar, 64 * s, slot, (int)w.h, page);
      }
    } else {
      for (uint32_t i = tid; i < halves * kKeys * NSLAB * 8; i += 64) {
        const uint32_t row = i / (NSLAB * 8), c = i % (NSLAB * 8), half = row / kKeys, in_half = row % kKeys;
        const uint32_t key = w.kt * kMassKeys + row;
        bool in = key < w.n && c * 8 < a.kv.D;
        const char* p = a.kv.k;
        if (in) {
          const uint32_t id = __ldg(ids + key / a.kv.B);
          in = id < a.kv.n_pages;
          if (in)
            p += 2 * (id * a.kv.ks_page + w.h * a.kv.ks_head + (int64_t)(key % a.kv.B) * a.kv.ks_slot + c * 8);
        }
        cp_async16(smem + (at * 2 + half) * Sh::kTile + (c / 8) * kSlab + in_half * 128 + (((c % 8) ^ (in_half & 7)) * 16), p, in);
      }
      cp_async_commit();
      cp_async_wait<0>();
      fence_async_shared();
      mbar_arrive(bar);
    }
  }
  return true;
}

template <typename T, int NSLAB, bool TMA>
__global__ void __launch_bounds__(kMassThreads, 1)
    k_mass_tiles(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mq, const AttnArgs a) {
  using Sh = MassShape<NSLAB>;
  extern __shared__ __align__(1024) char smem_raw[];
  MassShared& sh = *reinterpret_cast<MassShared*>(smem_raw + Sh::kRest);
  const uint32_t smem = smem_u32(smem_raw);
  const uint32_t warp = threadIdx.x >> 5;
  if (smem & 1023) {  // swizzled tiles start at whole groups of 8 rows
    if (threadIdx.x == 0) report(a.status, PTC_ERR_CUDA);
    return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sh.k_full[i]), TMA ? 1 : 64);
      mbar_init(smem_u32(&sh.k_empty[i]), 1);
    }
    for (uint32_t i = 0; i < kQueryRing; ++i) {
      mbar_init(smem_u32(&sh.q_full[i]), 1);
      mbar_init(smem_u32(&sh.q_empty[i]), 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(smem_u32(&sh.s_full[i]), 1);
      mbar_init(smem_u32(&sh.s_empty[i]), 8);
    }
    mbar_init(smem_u32(&sh.drain), 1);
    fence_mbar_init();
  }
  if (warp == 16) tmem_alloc(smem_u32(&sh.tmem), 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  grid_dep_sync();
  bool fine = true;
  if (a.plan[1].ok) {
    uint32_t segs = 0, units = 0;
    if (warp < 16) {
      fine = mass_sums(a, sh, warp / 4);
    } else if (warp == 16) {
      fine = mass_products<T, NSLAB>(a, sh, smem);
      // every product and every arrival it owes is done before the CTA ends
      if (elect_lane()) mma_commit(smem_u32(&sh.drain));
      __syncwarp();
      fine &= mbar_wait(smem_u32(&sh.drain), 0);
    } else if (warp == 18) {
      fine = mass_queries<NSLAB>(a, sh, &mq, smem, units);
      // copies in flight land before the CTA ends, whoever has given up
      for (uint32_t u = units > kQueryRing ? units - kQueryRing : 0; u < units; ++u)
        (void)mbar_wait(smem_u32(&sh.q_full[u % kQueryRing]), (u / kQueryRing) & 1);
    } else if (warp == 17 || !TMA) {
      fine = mass_keys<NSLAB, TMA>(a, sh, &mk, smem, segs);
      if (TMA)
        for (uint32_t k = segs > 2 ? segs - 2 : 0; k < segs; ++k)
          (void)mbar_wait(smem_u32(&sh.k_full[k & 1]), (k >> 1) & 1);
    }
  }
  if (!fine) report(a.status, PTC_ERR_TIMEOUT);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 16) tmem_free(sh.tmem, 512);
}

// blockIdx.y = 0: the key tiles that CTAs of the kernel above share, as
// the tile kernel does it for query tiles.  1: what no unit covers, the slots
// past every request's tokens, the requests without queries and the slots of
// no request.
__global__ void __launch_bounds__(kMassKeys) k_mass_join(const AttnArgs a) {
  grid_dep_sync();
  const AttnPlan* plan = a.plan + 1;
  if (!plan->ok) return;
  const uint32_t c = blockIdx.x, tid = threadIdx.x;
  if (blockIdx.y == 1) {
    for (uint64_t p = c; p < (uint64_t)a.kv.n_req * a.kv.H; p += gridDim.x) {
      const uint32_t r = (uint32_t)(p / a.kv.H), h = (uint32_t)(p % a.kv.H);
      const uint64_t at = h * a.mass_stride + a.kv.page_off[r] * a.kv.B, n = a.kv.kv_len[r];
      const uint64_t room = (a.kv.page_off[r + 1] - a.kv.page_off[r]) * a.kv.B;
      for (uint64_t j = (a.tok_off[r] == a.tok_off[r + 1] ? 0 : n) + tid; j < room; j += kMassKeys)
        a.mass_out[at + j] = j < n && a.mass_in ? a.mass_in[at + j] : 0.f;
    }
    const uint64_t lo = a.kv.page_off[0] * a.kv.B, hi = a.kv.page_off[a.kv.n_req] * a.kv.B;
    const uint64_t none = lo + a.kv.n_page_ids * a.kv.B - hi;  // slots of no request
    for (uint64_t i = (uint64_t)c * kMassKeys + tid; i < none * a.kv.H; i += (uint64_t)gridDim.x * kMassKeys) {
      const uint64_t h = i / none, x = i - h * none;
      copy_weight(a, h * a.mass_stride + (x < lo ? x : hi + x - lo));
    }
    return;
  }
  const CtaStart s = plan->start[c];
  if (s.u == plan->start[c + 1].u || s.minor == 0) return;
  const uint32_t m = (uint32_t)(a.tok_off[s.r + 1] - a.tok_off[s.r]), n = a.kv.kv_len[s.r];
  const uint64_t first = s.u - s.minor - kMassExtra;
  const Sharers sh = sharers(plan, a.ctas, first, first + kMassExtra + div_up(m, a.tq) - first_seeing(m, n, a.tq, s.major));
  for (uint32_t x = sh.c0 + 1; x < c; ++x)
    if (plan->start[x].u < plan->start[x + 1].u) return;  // not the first cut
  const uint64_t key = (uint64_t)s.major * kMassKeys + tid;
  if (key >= n) return;
  float sum = 0.f;
  for (uint32_t x = sh.c0; x <= sh.c1; ++x) {
    if (x != sh.c0 && plan->start[x].u == plan->start[x + 1].u) continue;
    sum += a.part_mass[(2 * (uint64_t)x + (x == sh.c0 && plan->start[x].u != first ? 1 : 0)) * kMassKeys + tid];
  }
  const uint64_t at = s.h * a.mass_stride + a.kv.page_off[s.r] * a.kv.B + key;
  a.mass_out[at] = (a.mass_in ? a.mass_in[at] : 0.f) + sum;
}

template <typename T, int NSLAB, bool TMA>
ptc_status launch_tiles(const AttnArgs& a, const CUtensorMap& mk, const CUtensorMap& mq, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  if (!large_smem(k_mass_tiles<T, NSLAB, TMA>, MassShape<NSLAB>::kSmem, ready)) return PTC_ERR_CUDA;
  PTC_KERNEL("k_mass_tiles", s, (k_mass_tiles<T, NSLAB, TMA>), a.ctas, kMassThreads, MassShape<NSLAB>::kSmem, mk, mq, a);
  return PTC_OK;
}

template <typename T>
ptc_status launch_by_tiles(const AttnArgs& a, const CUtensorMap& mk, const CUtensorMap& mq, bool tma, cudaStream_t s) {
  if (a.kv.D > 64) return tma ? launch_tiles<T, 2, true>(a, mk, mq, s) : launch_tiles<T, 2, false>(a, mk, mq, s);
  return tma ? launch_tiles<T, 1, true>(a, mk, mq, s) : launch_tiles<T, 1, false>(a, mk, mq, s);
}

}  // namespace

ptc_status launch_mass(const AttnArgs& a, bool bf16, const CUtensorMap& mk, const CUtensorMap& mq, bool tma,
                       cudaStream_t s) {
  if (a.scores || a.n_tok == 0) {
    const uint64_t slots = a.kv.n_page_ids * a.kv.B;
    PTC_KERNEL("k_mass_rows", s, k_mass_rows, dim3((uint32_t)((slots + kRowSlots - 1) / kRowSlots), a.kv.H), kRowThreads, 0,
               a);
    return PTC_OK;
  }
  const ptc_status st = bf16 ? launch_by_tiles<__nv_bfloat16>(a, mk, mq, tma, s) : launch_by_tiles<__half>(a, mk, mq, tma, s);
  if (st != PTC_OK) return st;
  PTC_KERNEL("k_mass_join", s, k_mass_join, dim3(a.ctas, 2), kMassKeys, 0, a);
  return PTC_OK;
}

}  // namespace ptc
