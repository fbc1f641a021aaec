// Attention over pages of 4 bits for requests of few query rows: single tokens,
// or a few of them.
//
// One pass over the keys and values, which HBM bounds if the instructions keep
// up: 6.6 TB/s are 44 values a cycle and SM, so a value has about three of a
// lane's instructions.  They become 16-bit numbers in the registers where the
// matrix instructions want them, with no way through shared memory in 16 bits
// (which tcgen05's operands need, 2 bytes written and read a value):
//   scores   S^T = K Q^T       16 keys x 8 query rows, mma.sync m16n8k16
//   softmax  running maximum and sum of a query row in 32 bits
//   values   O^T += V^T P^T    16 channels x 8 query rows, 16 keys at a time
// A word of codes is eight neighbouring channels of a key, even ones in its low
// half, so a shifted and masked word is two channels as K's operand wants them;
// the low (high) halves of two keys' words together are one channel of both, as
// V^T's operand does.  Eight query rows are all that an instruction's N asks for.
//
// A call's units are 128 keys of a request's key head, and `kExtra` for what a
// head's tile costs by itself.  CTA c of C has the units from U c / C on, so where
// a cut lies, and which CTAs share a tile, is arithmetic that every CTA does for
// itself from the requests' lengths; there is no plan to wait for.  Warp 8 copies
// units into a ring, warps 0-7 take 16 keys of each; at the tile's end they put
// their rows together, and of a split tile the last CTA that is done does so with
// the parts.
#include "ptc_attn4.cuh"

namespace ptc {
namespace {

constexpr uint32_t kUnit = 128, kWarps = 8, kThreads = 32 * (kWarps + 1);
constexpr uint32_t kExtra = 2;
constexpr float kMove4 = 256.f;  // the maximum moves when a weight passes this

template <typename T>
struct Mma16;
template <>
struct Mma16<__nv_bfloat16> {
  static constexpr float kShift = 0.f, kScale = 1.f;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  static __device__ __forceinline__ void run(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                             uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};
// (weights of fp16 caches are scaled by 2^7: small ones would fall among fp16's subnormals)
template <>
struct Mma16<__half> {
  static constexpr float kShift = 7.f, kScale = 128.f;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 x = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
  }
  static __device__ __forceinline__ void run(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                             uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};
// An 8 x 8 matrix of 16-bit numbers over a warp, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// The eight warps of the products.
__device__ __forceinline__ void warps_sync() { asm volatile("bar.sync 1, 256;" ::: "memory"); }

// NS: rows of 64 or 128 channels.  NT: eight or sixteen query rows.
template <int NS, int NT>
struct Shape {
  static constexpr uint32_t kDim = 64 * NS, kRow = NS == 1 ? 48 : 80, kQRows = 8 * NT;
  static constexpr uint32_t kTensor = kUnit * kRow, kStage = 2 * kTensor;
  static constexpr uint32_t kCtas = NS * NT <= 2 ? 2 : 1;  // of an SM: by their registers
  static constexpr uint32_t kRing = NS == 1 ? 4 : NT == 1 ? 3 : 6;
  static constexpr uint32_t kORow = kDim + 4;  // 32-bit words of a row on its way to the other warps
  static constexpr uint32_t kBytes = kRing * kStage + kWarps * kQRows * kORow * 4;
};

struct Shared {
  uint64_t full[8], empty[8];
  uint64_t off[257];  // units before a block of requests
  uint64_t tok0[256], page0[256];
  uint32_t m[256], n[256];
  uint64_t warp_sum[8];
  float2 ml[kWarps][kFew4Rows];
  uint32_t last;
};

__device__ __forceinline__ uint32_t tiles_of(uint32_t n) { return n ? (n - 1) / kUnit + 1 : 1; }
__device__ __forceinline__ uint64_t units_of(const Few4Args& a, uint32_t m, uint32_t n) {
  return m ? (uint64_t)a.kv.H * (tiles_of(n) + kExtra) : 0;
}

// A CTA's way through its units: tile by tile, keys [kv0, kv1) times 128 of each.
struct Way {
  uint64_t end, tile0, tok0, page0;  // unit after the CTA's last, the tile's first
  uint32_t r, h, m, n, tiles, kv0, kv1;

  __device__ __forceinline__ void request(const Few4Args& a, const Shared& sh) {
    if (a.kv.n_req <= 256) {
      m = sh.m[r];
      n = sh.n[r];
      tok0 = sh.tok0[r];
      page0 = sh.page0[r];
    } else {
      tok0 = a.tok_off[r];
      m = (uint32_t)(a.tok_off[r + 1] - tok0);
      n = a.kv.kv_len[r];
      page0 = a.kv.page_off[r];
    }
    tiles = tiles_of(n);
  }
  // The CTA's keys of the tile at hand; false if it has none.
  __device__ __forceinline__ bool keys(uint64_t from) {
    const uint64_t first = tile0 + kExtra;
    kv0 = from > first ? (uint32_t)(from - first) : 0;
    kv1 = end <= first ? 0 : end - first < tiles ? (uint32_t)(end - first) : tiles;
    return kv0 < kv1;
  }
  __device__ __forceinline__ bool begin(const Few4Args& a, const Shared& sh, uint64_t all, uint32_t c, uint32_t ctas) {
    const uint64_t u = all * c / ctas;
    end = all * (c + 1) / ctas;
    if (u >= end) return false;
    uint32_t lo = 0, hi = 255;
    while (lo < hi) {
      const uint32_t mid = (lo + hi + 1) / 2;
      if (sh.off[mid] <= u) lo = mid;
      else hi = mid - 1;
    }
    uint64_t off = sh.off[lo];
    r = lo;
    if (a.kv.n_req > 256) {  // a block of requests, 32 at a time
      const uint32_t per = (a.kv.n_req + 255) / 256, lane = threadIdx.x & 31;
      for (uint32_t r0 = lo * per;; r0 += 32) {
        const uint32_t x = r0 + lane;
        uint64_t mine = 0;
        if (x < a.kv.n_req && x < (lo + 1) * per) mine = units_of(a, (uint32_t)(a.tok_off[x + 1] - a.tok_off[x]), a.kv.kv_len[x]);
        uint64_t incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint64_t y = __shfl_up_sync(kFull, incl, o);
          if (lane >= (uint32_t)o) incl += y;
        }
        const uint32_t here = __ballot_sync(kFull, u < off + incl);
        if (here) {
          const int src = __ffs(here) - 1;
          r = r0 + src;
          off += __shfl_sync(kFull, incl - mine, src);
          break;
        }
        off += __shfl_sync(kFull, incl, 31);
        if (r0 + 32 >= (lo + 1) * per) return false;  // (the lists are sound, so this is not reached)
      }
    }
    request(a, sh);
    const uint32_t each = tiles + kExtra;
    h = (uint32_t)((u - off) / each);
    tile0 = off + (uint64_t)h * each;
    return keys(u) || next(a, sh);
  }
  __device__ __forceinline__ bool next(const Few4Args& a, const Shared& sh) {
    tile0 += tiles + kExtra;
    if (tile0 + kExtra >= end) return false;
    if (++h == a.kv.H) {
      h = 0;
      do {
        if (++r >= a.kv.n_req) return false;
        request(a, sh);
      } while (m == 0);
    }
    return keys(0);
  }
};

// What a call's requests have of units, and whether its lists are sound.  By the
// whole CTA; request r is of block r / per.
__device__ __forceinline__ bool add_up(const Few4Args& a, Shared& sh, uint64_t& all) {
  const uint32_t tid = threadIdx.x, lane = tid & 31, R = a.kv.n_req, per = (R + 255) / 256;
  bool bad = tid == 0 && (a.tok_off[0] != 0 || a.tok_off[R] != a.n_tok);
  uint64_t mine = 0, incl = 0;
  if (tid < 256) {
    for (uint32_t r = tid * per; r < (tid + 1) * per && r < R; ++r) {
      const uint64_t lo = a.tok_off[r], hi = a.tok_off[r + 1];
      const uint32_t n = a.kv.kv_len[r];
      const bool wrong = (lo > hi) | (hi > a.n_tok) | (hi - lo > a.max_q_len) | !pages_hold(a.kv, r, n) | (n > kMost4);
      bad |= wrong;
      const uint32_t m = wrong ? 0 : (uint32_t)(hi - lo);
      mine += units_of(a, m, n);
      if (per == 1) {
        sh.tok0[r] = lo;
        sh.page0[r] = a.kv.page_off[r];
        sh.m[r] = m;
        sh.n[r] = n;
      }
    }
    incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t y = __shfl_up_sync(kFull, incl, o);
      if (lane >= (uint32_t)o) incl += y;
    }
    if (lane == 31) sh.warp_sum[tid / 32] = incl;
  }
  bad = __syncthreads_or(bad);
  uint64_t before = 0;
  all = 0;
#pragma unroll
  for (uint32_t x = 0; x < 8; ++x) {
    if (x < tid / 32) before += sh.warp_sum[x];
    all += sh.warp_sum[x];
  }
  if (tid < 256) sh.off[tid] = before + incl - mine;
  if (bad && blockIdx.x == 0 && tid == 0) report(a.status, PTC_ERR_INVALID_ARG);
  __syncthreads();
  return !bad;
}

// Units into the ring, by tensor copies of `box` slots (a divisor of the page
// size and of a unit).  Slots of no page read as zeros: their page's coordinate is
// n_pages, out of range.  The pages of the unit after are asked for meanwhile.
template <int NS, int NT>
__device__ __forceinline__ bool copy_units(const Few4Args& a, Shared& sh, Way& w, bool more, uint32_t ring,
                                           const CUtensorMap* mk, const CUtensorMap* mv, uint32_t& issued) {
  using S = Shape<NS, NT>;
  const uint32_t lane = threadIdx.x & 31, boxes = kUnit / a.box;
  uint32_t j = w.kv0, id = 0, slot = 0, head = 0;
  bool in = false;
  auto ask = [&] {
    const uint32_t key = j * kUnit + lane * a.box, at = key / a.kv.B;
    in = lane < boxes && key < w.n;
    slot = key - at * a.kv.B;
    head = w.h;
    id = in ? __ldg(a.kv.page_ids + w.page0 + at) : 0;
  };
  if (more) ask();
  while (more) {
    int page = (int)a.kv.n_pages;
    if (in && id < a.kv.n_pages) page = (int)id;
    else if (in) report(a.status, PTC_ERR_INVALID_ARG);
    const int s0 = in ? (int)slot : 0, h0 = (int)head;
    if (++j == w.kv1) {
      more = w.next(a, sh);
      j = w.kv0;
    }
    if (more) ask();
    const uint32_t at = issued % S::kRing;
    if (issued >= S::kRing && !mbar_wait(smem_u32(&sh.empty[at]), (issued / S::kRing - 1) & 1, a.limit)) return false;
    ++issued;
    const uint32_t bar = smem_u32(&sh.full[at]), dst = ring + at * S::kStage + lane * a.box * S::kRow;
    if (lane == 0) mbar_expect(bar, S::kStage);
    __syncwarp();
    if (lane < boxes) {
      tma_load_4d(dst, mk, bar, 0, s0, h0, page);
      tma_load_4d(dst + S::kTensor, mv, bar, 0, s0, h0, page);
    }
  }
  return true;
}

// The same for page sizes that are no multiple of 8, 16 bytes a copy.
template <int NS, int NT>
__device__ __forceinline__ bool gather_units(const Few4Args& a, Shared& sh, Way& w, bool more, uint32_t ring, uint32_t& issued) {
  using S = Shape<NS, NT>;
  constexpr uint32_t kPieces = S::kRow / 16;
  const uint32_t lane = threadIdx.x & 31;
  for (; more; more = w.next(a, sh)) {
    const uint32_t* ids = a.kv.page_ids + w.page0;
    for (uint32_t j = w.kv0; j < w.kv1; ++j) {
      const uint32_t at = issued % S::kRing;
      if (issued >= S::kRing && !mbar_wait(smem_u32(&sh.empty[at]), (issued / S::kRing - 1) & 1, a.limit)) return false;
      ++issued;
      for (uint32_t x = 0; x < kUnit; x += 32) {
        const uint32_t row = x + lane, key = j * kUnit + row, page = key / a.kv.B, slot = key - page * a.kv.B;
        bool in = key < w.n;
        uint32_t id = 0;
        if (in) {
          id = __ldg(ids + page);
          if (id >= a.kv.n_pages) {
            report(a.status, PTC_ERR_INVALID_ARG);
            in = false;
          }
        }
        const char* k = in ? a.kv.k + id * a.kv.ks_page + w.h * a.kv.ks_head + slot * a.kv.ks_slot : a.kv.k;
        const char* v = in ? a.kv.v + id * a.kv.vs_page + w.h * a.kv.vs_head + slot * a.kv.vs_slot : a.kv.v;
        const uint32_t dst = ring + at * S::kStage + row * S::kRow;
#pragma unroll
        for (uint32_t p = 0; p < kPieces; ++p) {
          cp_async16(dst + 16 * p, k + 16 * p, in);
          cp_async16(dst + S::kTensor + 16 * p, v + 16 * p, in);
        }
      }
      asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&sh.full[at])) : "memory");
    }
  }
  return true;
}

__device__ __forceinline__ uint32_t lds32(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  return x;
}
// NS * 2 words.
template <int NS>
__device__ __forceinline__ void lds_words(uint32_t (&x)[2 * NS], uint32_t at) {
  if constexpr (NS == 2)
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(at) : "memory");
  else
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x[0]), "=r"(x[1]) : "r"(at) : "memory");
}
template <int NS>
__device__ __forceinline__ void lds_half(uint32_t (&x)[NS], uint32_t at) {
  if constexpr (NS == 2)
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x[0]), "=r"(x[1]) : "r"(at) : "memory");
  else
    x[0] = lds32(at);
}

// A warp's rows so far: of query rows 8 i + 2 t and 8 i + 2 t + 1 (t = lane % 4), the
// maximum (as a power of two), the lane's share of the sum, and channels.
template <int NS, int NT>
struct Rows {
  float top[NT][2], l[NT][2], o[NT][4 * NS][4];
};

// 16 keys of a unit.  Row i of the matrices is key (2 (i % 8 / 2) + 4 (i % 2)) % 8 +
// 8 (i % 2) + i / 8: rows of 80 (48) bytes in that order meet no bank twice, neither
// where four lanes read K's rows whole nor where eight read a piece of V's each.
template <typename T, int NS, int NT>
__device__ __forceinline__ void take_keys(uint32_t at, uint32_t key0, uint32_t n, const int32_t (&see)[NT][2], int32_t least,
                                          float sl2, const uint32_t (&q)[NT][8 * NS], Rows<NS, NT>& st) {
  using S = Shape<NS, NT>;
  using M = Mma16<T>;
  const uint32_t lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  // scores
  const uint32_t kg = ((g & 6) + 4 * (g & 1) & 7) + 8 * (g & 1);
  const uint32_t k_at = at + kg * S::kRow;
  uint32_t wa[2 * NS], wb[2 * NS];
  lds_words<NS>(wa, k_at + 8 * NS * t);
  lds_words<NS>(wb, k_at + S::kRow + 8 * NS * t);
  const uint32_t group = NS == 2 ? t : t >> 1;
  const uint32_t pa = lds32(k_at + 32 * NS + 4 * group), pb = lds32(k_at + S::kRow + 32 * NS + 4 * group);
  const uint32_t sa = both_low(pa), ba = both_high(pa), sb = both_low(pb), bb = both_high(pb);
  float s[NT][4];
#pragma unroll
  for (int x = 0; x < NT; ++x)
#pragma unroll
    for (int k = 0; k < 4; ++k) s[x][k] = 0.f;
#pragma unroll
  for (int i = 0; i < 2 * NS; ++i)
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      const uint32_t a0 = fma16x2<T>(pair4<T>(wa[i], j), sa, ba), a1 = fma16x2<T>(pair4<T>(wb[i], j), sb, bb);
      const uint32_t a2 = fma16x2<T>(pair4<T>(wa[i], j + 1), sa, ba), a3 = fma16x2<T>(pair4<T>(wb[i], j + 1), sb, bb);
#pragma unroll
      for (int x = 0; x < NT; ++x) M::run(s[x], a0, a1, a2, a3, q[x][4 * i + j], q[x][4 * i + j + 1]);
    }
  // weights; s[x][0], s[x][1]: key kg of query rows 2 t and 2 t + 1, [2], [3]: the key after
  if ((int32_t)(key0 + 16) > least) {
    const int32_t key = (int32_t)(key0 + kg);
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (key + (k >> 1) >= see[x][k & 1]) s[x][k] = -INFINITY;
  }
  float p[NT][4];
  bool move = false;
  auto weigh = [&] {
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float sub = (st.top[x][k & 1] == -INFINITY ? 0.f : st.top[x][k & 1]) - M::kShift;
        p[x][k] = exp2_approx(fmaf(s[x][k], sl2, -sub));
        move |= !(p[x][k] <= kMove4 * M::kScale) | (st.top[x][k & 1] == -INFINITY && s[x][k] != -INFINITY);
      }
  };
  weigh();
  if (__any_sync(kFull, move)) {
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        float mx = fmaxf(s[x][y], s[x][y + 2]) * sl2;
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) mx = fmaxf(mx, __shfl_xor_sync(kFull, mx, o));
        const float top = st.top[x][y], up = fmaxf(top, mx), f = top == -INFINITY ? 0.f : exp2_approx(top - up);
        st.top[x][y] = up;
        st.l[x][y] *= f;
#pragma unroll
        for (int i = 0; i < 4 * NS; ++i) {
          st.o[x][i][y] *= f;
          st.o[x][i][y + 2] *= f;
        }
      }
    weigh();
  }
  uint32_t b[NT][2];
#pragma unroll
  for (int x = 0; x < NT; ++x) {
    st.l[x][0] += p[x][0] + p[x][2];
    st.l[x][1] += p[x][1] + p[x][3];
    b[x][0] = transposed(M::pack(p[x][0], p[x][1]));
    b[x][1] = transposed(M::pack(p[x][2], p[x][3]));
  }
  // values: keys 2 t and 2 t + 1 of the matrix's order, and the two 8 rows on
  const uint32_t r0 = 2 * t, r1 = ((2 * t + 4) & 7) + 8;
  const uint32_t v0 = at + S::kTensor + r0 * S::kRow, v1 = at + S::kTensor + r1 * S::kRow;
  uint32_t w[4][NS], par[4];
  const uint32_t v_group = NS == 2 ? g >> 1 : g >> 2;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t row = (k & 1 ? v1 : v0) + (k >> 1) * S::kRow;
    lds_half<NS>(w[k], row + 4 * NS * g);
    par[k] = lds32(row + 32 * NS + 4 * v_group);
  }
  if (key0 + 16 > n) {  // slots that hold no token may hold anything: values of 0
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (key0 + (k & 1 ? r1 : r0) + (k >> 1) >= n) par[k] = 0;
  }
  const uint32_t s0 = __byte_perm(par[0], par[1], 0x5410), b0 = __byte_perm(par[0], par[1], 0x7632);
  const uint32_t s1 = __byte_perm(par[2], par[3], 0x5410), b1 = __byte_perm(par[2], par[3], 0x7632);
#pragma unroll
  for (int i = 0; i < NS; ++i) {
    const uint32_t e0 = __byte_perm(w[0][i], w[1][i], 0x5410), d0 = __byte_perm(w[0][i], w[1][i], 0x7632);
    const uint32_t e1 = __byte_perm(w[2][i], w[3][i], 0x5410), d1 = __byte_perm(w[2][i], w[3][i], 0x7632);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t a0 = fma16x2<T>(pair4<T>(e0, j), s0, b0), a1 = fma16x2<T>(pair4<T>(d0, j), s0, b0);
      const uint32_t a2 = fma16x2<T>(pair4<T>(e1, j), s1, b1), a3 = fma16x2<T>(pair4<T>(d1, j), s1, b1);
#pragma unroll
      for (int x = 0; x < NT; ++x) M::run(st.o[x][4 * i + j], a0, a1, a2, a3, b[x][0], b[x][1]);
    }
  }
}

// A row's parts put together, `count` of them: part p is at slot(p).  By a warp.
template <typename T, int NS, int NT>
__device__ __noinline__ void join_row(const Few4Args& a, uint32_t c0, uint32_t count, uint32_t row, uint64_t at) {
  using S = Shape<NS, NT>;
  const uint32_t lane = threadIdx.x & 31, D = a.kv.D;
  auto slot = [&](uint32_t p) { return 2 * (uint64_t)(c0 + p) + (p == 0 ? 1 : 0); };
  float top = -INFINITY, l = 0.f;
  for (uint32_t p = lane; p < count; p += 32) top = fmaxf(top, __ldcg(a.part_ml + slot(p) * S::kQRows + row).x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
  float4 o4 = make_float4(0.f, 0.f, 0.f, 0.f);
  const bool in = 4 * lane < S::kDim;
  for (uint32_t p0 = 0; p0 < count; p0 += 32) {
    float f = 0.f;
    if (p0 + lane < count) {
      const float2 ml = __ldcg(a.part_ml + slot(p0 + lane) * S::kQRows + row);
      f = ml.x == -INFINITY ? 0.f : exp2_approx(ml.x - top);
      l += ml.x == -INFINITY ? 0.f : ml.y * f;
    }
    const uint32_t some = count - p0 < 32 ? count - p0 : 32;
#pragma unroll 8
    for (uint32_t p = 0; p < some; ++p) {
      const float4 x = in ? __ldcg(reinterpret_cast<const float4*>(a.part + (slot(p0 + p) * S::kQRows + row) * S::kDim) + lane)
                          : make_float4(0.f, 0.f, 0.f, 0.f);
      const float fp = __shfl_sync(kFull, f, p);
      if (fp == 0.f) continue;  // the row saw no key of the part
      o4.x = fmaf(x.x, fp, o4.x);
      o4.y = fmaf(x.y, fp, o4.y);
      o4.z = fmaf(x.z, fp, o4.z);
      o4.w = fmaf(x.w, fp, o4.w);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(kFull, l, o);
  const bool none = top == -INFINITY;
  const float inv = none ? 0.f : 1.f / l;
  if (4 * lane < D)
    *reinterpret_cast<uint2*>(a.out + 2 * (at * D + 4 * lane)) =
        make_uint2(Mma16<T>::pack(o4.x * inv, o4.y * inv), Mma16<T>::pack(o4.z * inv, o4.w * inv));
  if (lane == 0) a.lse[at] = none ? -INFINITY : (top + log2_approx(l)) * kLn2;
}

template <typename T, int NS, int NT>
__device__ __forceinline__ bool product_warps(const Few4Args& a, Shared& sh, Way& w, bool more, uint32_t ring, float* rows,
                                              uint64_t all, uint32_t ctas) {
  using S = Shape<NS, NT>;
  using M = Mma16<T>;
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const uint32_t D = a.kv.D, G = a.G;
  const float sl2 = a.scale * kLog2e;
  bool alive = true;  // a warp that has given up waiting runs on without, for the others at the barriers
  uint32_t item = 0;
  for (; more; more = w.next(a, sh)) {
    // the queries' operand: row 8 x + g, channels 16 NS t on
    uint32_t q[NT][8 * NS];
    int32_t see[NT][2], least = (int32_t)w.n;
#pragma unroll
    for (int x = 0; x < NT; ++x) {
      const uint32_t i = 8 * x + g, tok = i / G, head = w.h * G + i % G;
      const char* row = a.q + 2 * ((int64_t)(w.tok0 + tok) * a.q_tok + (int64_t)head * a.q_head);
#pragma unroll
      for (uint32_t k = 0; k < 2 * NS; ++k) {
        const uint32_t d = 16 * NS * t + 8 * k;
        uint4 y = make_uint4(0, 0, 0, 0);
        if (tok < w.m && d < D) y = *reinterpret_cast<const uint4*>(row + 2 * d);
        q[x][4 * k] = y.x;
        q[x][4 * k + 1] = y.y;
        q[x][4 * k + 2] = y.z;
        q[x][4 * k + 3] = y.w;
      }
#pragma unroll
      for (uint32_t y = 0; y < 2; ++y) {  // keys that query row 8 x + 2 t + y sees (rows that are none: all)
        const uint32_t mine = (8 * x + 2 * t + y) / G;
        const int64_t last = (int64_t)w.n - w.m + mine + 1;
        see[x][y] = mine >= w.m ? (int32_t)w.n : last > 0 ? (int32_t)last : 0;
      }
      const int64_t first = (int64_t)w.n - w.m + 1;
      least = first > 0 ? (int32_t)first : 0;
    }
    Rows<NS, NT> st;
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        st.top[x][y] = -INFINITY;
        st.l[x][y] = 0.f;
#pragma unroll
        for (int i = 0; i < 4 * NS; ++i) st.o[x][i][y] = st.o[x][i][y + 2] = 0.f;
      }
    for (uint32_t j = w.kv0; j < w.kv1; ++j, ++item) {
      const uint32_t at = item % S::kRing, key0 = j * kUnit + 16 * warp;
      if (alive) alive = mbar_wait(smem_u32(&sh.full[at]), (item / S::kRing) & 1, a.limit);
      if (key0 < w.n) take_keys<T, NS, NT>(ring + at * S::kStage + 16 * warp * S::kRow, key0, w.n, see, least, sl2, q, st);
      mbar_arrive_warp(smem_u32(&sh.empty[at]));
    }
    // the warps' rows
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        float l = st.l[x][y];
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l += __shfl_xor_sync(kFull, l, o);
        const uint32_t i = 8 * x + 2 * t + y;
        if (g == 0) sh.ml[warp][i] = make_float2(l != 0.f ? st.top[x][y] - M::kShift : -INFINITY, l);
        float4* to = reinterpret_cast<float4*>(rows + (warp * S::kQRows + i) * S::kORow + 8 * NS * g);
#pragma unroll
        for (int k = 0; k < 2 * NS; ++k)
          to[k] = make_float4(st.o[x][2 * k][y], st.o[x][2 * k][y + 2], st.o[x][2 * k + 1][y], st.o[x][2 * k + 1][y + 2]);
      }
    warps_sync();
    const bool whole = w.kv0 == 0 && w.kv1 == w.tiles;
    const uint32_t used = w.m * G;
    const uint64_t out0 = w.tok0 * a.n_q_heads + w.h * G;  // of row 0; row i is token i / G, head i % G
    const uint64_t slot = 2 * (uint64_t)blockIdx.x + (w.kv0 ? 0 : 1);
    constexpr uint32_t kAcross = S::kDim / 4;
    for (uint32_t e = tid; e < S::kQRows * kAcross; e += 32 * kWarps) {
      const uint32_t i = e / kAcross, c = 4 * (e % kAcross);
      if (i >= used) break;
      float top = -INFINITY, l = 0.f;
#pragma unroll
      for (uint32_t x = 0; x < kWarps; ++x) top = fmaxf(top, sh.ml[x][i].x);
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (uint32_t x = 0; x < kWarps; ++x) {
        const float2 ml = sh.ml[x][i];
        if (ml.x == -INFINITY) continue;
        const float f = exp2_approx(ml.x - top);
        const float4 y = *reinterpret_cast<const float4*>(rows + (x * S::kQRows + i) * S::kORow + c);
        l = fmaf(ml.y, f, l);
        o.x = fmaf(y.x, f, o.x);
        o.y = fmaf(y.y, f, o.y);
        o.z = fmaf(y.z, f, o.z);
        o.w = fmaf(y.w, f, o.w);
      }
      if (whole) {
        const bool none = top == -INFINITY;
        const float inv = none ? 0.f : 1.f / l;
        const uint64_t to = out0 + (uint64_t)(i / G) * a.n_q_heads + i % G;
        if (c < D)
          *reinterpret_cast<uint2*>(a.out + 2 * (to * D + c)) =
              make_uint2(M::pack(o.x * inv, o.y * inv), M::pack(o.z * inv, o.w * inv));
        if (c == 0) a.lse[to] = none ? -INFINITY : (top + log2_approx(l)) * kLn2;
      } else {
        *reinterpret_cast<float4*>(a.part + (slot * S::kQRows + i) * S::kDim + c) = o;
        if (c == 0) a.part_ml[slot * S::kQRows + i] = make_float2(top, l);
      }
    }
    if (!whole) {
      // the CTAs that share the tile: those of its first and its last key, and all between
      const uint64_t first = w.tile0 + kExtra;
      const uint32_t c0 = (uint32_t)(((first + 1) * ctas + all - 1) / all - 1);
      const uint32_t c1 = (uint32_t)(((first + w.tiles) * ctas + all - 1) / all - 1);
      __threadfence();
      warps_sync();
      if (tid == 0) sh.last = atomicAdd(a.arrived + c0, 1u) == c1 - c0;
      warps_sync();
      if (sh.last) {
        __threadfence();
        for (uint32_t i = warp; i < used; i += kWarps)
          join_row<T, NS, NT>(a, c0, c1 - c0 + 1, i, out0 + (uint64_t)(i / G) * a.n_q_heads + i % G);
      }
    }
    warps_sync();
  }
  return alive;
}

template <typename T, int NS, int NT, bool TMA>
__global__ void __launch_bounds__(kThreads, Shape<NS, NT>::kCtas)
    k_attn4_few(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, const __grid_constant__ Few4Args a) {
  using S = Shape<NS, NT>;
  extern __shared__ __align__(1024) char smem_raw[];
  __shared__ Shared sh;
  const uint32_t ring = smem_u32(smem_raw), warp = threadIdx.x >> 5;
  float* rows = reinterpret_cast<float*>(smem_raw + S::kRing * S::kStage);
  if (ring & 127) {  // tensor copies land on whole lines
    if (threadIdx.x == 0) report(a.status, PTC_ERR_CUDA);
    return;
  }
  if (threadIdx.x == 0) {
    for (uint32_t i = 0; i < S::kRing; ++i) {
      mbar_init(smem_u32(&sh.full[i]), TMA ? 1 : 32);
      mbar_init(smem_u32(&sh.empty[i]), kWarps);
    }
    fence_mbar_init();
  }
  grid_dep_sync();
  uint64_t all;
  if (!add_up(a, sh, all)) return;
  const uint32_t ctas = all < a.ctas ? (uint32_t)all : a.ctas;  // every CTA has a unit
  if (blockIdx.x >= ctas) return;
  Way w;
  const bool more = w.begin(a, sh, all, blockIdx.x, ctas);
  bool fine = true;
  uint32_t issued = 0;
  if (warp < kWarps) {
    fine = product_warps<T, NS, NT>(a, sh, w, more, ring, rows, all, ctas);
  } else if (!a.withhold) {
    fine = TMA ? copy_units<NS, NT>(a, sh, w, more, ring, &mk, &mv, issued) : gather_units<NS, NT>(a, sh, w, more, ring, issued);
    if (!TMA) {
      cp_async_commit();
      cp_async_wait<0>();
    }
  }
  if (!fine) report(a.status, PTC_ERR_TIMEOUT);
  // Where a role has given up, the copies that were issued land before the CTA ends.
  if (__syncthreads_or(!fine) && warp == kWarps && TMA)
    for (uint32_t i = issued > S::kRing ? issued - S::kRing : 0; i < issued; ++i)
      (void)mbar_wait(smem_u32(&sh.full[i % S::kRing]), (i / S::kRing) & 1);
}

template <typename T, int NS, int NT, bool TMA>
ptc_status launch_one(const Few4Args& a, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t s) {
  constexpr int smem = Shape<NS, NT>::kBytes;
  static std::atomic<uint64_t> ready{0};
  const auto kernel = k_attn4_few<T, NS, NT, TMA>;
  if (!large_smem(kernel, smem, ready)) return PTC_ERR_CUDA;
  PTC_KERNEL("k_attn4_few", s, kernel, a.ctas, kThreads, smem, mk, mv, a);
  return PTC_OK;
}
template <typename T>
ptc_status launch_some(const Few4Args& a, uint32_t rows, bool tma, const CUtensorMap& mk, const CUtensorMap& mv, cudaStream_t s) {
  const bool wide = a.kv.D > 64, two = rows > 8;
#define PTC_FEW4(NS, NT) (tma ? launch_one<T, NS, NT, true>(a, mk, mv, s) : launch_one<T, NS, NT, false>(a, mk, mv, s))
  return wide ? two ? PTC_FEW4(2, 2) : PTC_FEW4(2, 1) : two ? PTC_FEW4(1, 2) : PTC_FEW4(1, 1);
#undef PTC_FEW4
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

uint32_t few4_ctas(uint32_t head_dim, uint32_t rows) {
  const uint32_t n = (uint32_t)num_sms() * (head_dim > 64 && rows > 8 ? 1 : 2);
  return n < kFew4MaxCtas ? n : kFew4MaxCtas;
}

size_t few4_ws(uint32_t head_dim, uint32_t rows) {
  const size_t places = 2 * (size_t)few4_ctas(head_dim, rows) * (rows > 8 ? 16 : 8);
  return up256(4 * kFew4MaxCtas) + up256(8 * places) + up256(4 * places * padded4(head_dim));
}

void few4_place(Few4Args& a, uint32_t rows, char* ws) {
  a.ctas = few4_ctas(a.kv.D, rows);
  const size_t places = 2 * (size_t)a.ctas * (rows > 8 ? 16 : 8);
  a.arrived = reinterpret_cast<uint32_t*>(ws);
  ws += up256(4 * kFew4MaxCtas);
  a.part_ml = reinterpret_cast<float2*>(ws);
  a.part = reinterpret_cast<float*>(ws + up256(8 * places));
}

ptc_status launch_few4(Few4Args& a, uint32_t rows, bool bf16, cudaStream_t s) {
  a.box = kUnit;
  while (a.kv.B % a.box) a.box /= 2;
  const bool tma = a.box >= 8 && a.kv.n_pages > 0;
  CUtensorMap mk = {}, mv = {};
  if (tma && (!cache4_map(&mk, a.kv, a.kv.k, a.kv.ks_page, a.kv.ks_head, a.kv.ks_slot, a.box) ||
              !cache4_map(&mv, a.kv, a.kv.v, a.kv.vs_page, a.kv.vs_head, a.kv.vs_slot, a.box)))
    return PTC_ERR_CUDA;
  const ptc_status st = fill_async(a.arrived, 0u, 4 * a.ctas, s);
  if (st != PTC_OK) return st;
  return bf16 ? launch_some<__nv_bfloat16>(a, rows, tma, mk, mv, s) : launch_some<__half>(a, rows, tma, mk, mv, s);
}

}  // namespace ptc
